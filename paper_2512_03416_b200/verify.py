"""Drafted tokens verified by sampling from the model's distributions (ts_verify_tokens). PyTorch supplies device memory and the
stream; all computation happens inside libtokenscale.so.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence

import torch

from . import binding as B
from .decoder import _check, _raw_stream


class Verified(NamedTuple):
    emitted: torch.Tensor        # int32 [N]: per request count tokens, then -1
    count: torch.Tensor          # int32 [requests]
    path: torch.Tensor           # int32 [N]: the rows of the nodes walked, count per request, then -1
    logprob: torch.Tensor        # float32 [N]: of the emitted tokens, then 0


def _rows(t: torch.Tensor, what: str, like: Optional[torch.Tensor] = None) -> None:
    if not t.is_cuda or t.dim() != 2 or t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{what} must be a bf16 or float32 CUDA tensor [rows, vocab]")
    if t.shape[1] < 1 or (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"the {what} of a row must lie next to each other, and rows may not overlap")
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{what} must be of the logits' shape, type and device")


def verify_tokens(logits: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor, n_nodes: Sequence[int], u_accept: torch.Tensor,
                  u_sample: torch.Tensor, draft: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                  draft_scale: Optional[torch.Tensor] = None) -> Verified:
    """logits (and draft, of the model that drew the drafts): bf16 or float32 [N, vocab], N the sum of n_nodes (1 to 64 per request). tokens,
    parents: int32 [N]; u_accept: float32 [N], u_sample: float32 [requests], from [0, 1); scale, draft_scale: float32 [N], inverse temperatures."""
    _rows(logits, "logits")
    dev, (n, vocab), requests = logits.device, logits.shape, len(n_nodes)
    if draft is not None:
        _rows(draft, "draft", logits)
    if sum(n_nodes) != n:
        raise ValueError(f"n_nodes adds up to {sum(n_nodes)}, the logits have {n} rows")
    for t, count, dtype, what in ((tokens, n, torch.int32, "tokens"), (parents, n, torch.int32, "parents"), (u_accept, n, torch.float32, "u_accept"),
                                  (u_sample, requests, torch.float32, "u_sample"), (scale, n, torch.float32, "scale"),
                                  (draft_scale, n, torch.float32, "draft_scale")):
        if t is not None and (t.dtype != dtype or t.device != dev or t.numel() != count or not t.is_contiguous()):
            raise ValueError(f"{what} must be a contiguous {str(dtype)[6:]} tensor of {count} values on {dev}")
    emitted, path = (torch.empty(n, dtype=torch.int32, device=dev) for _ in range(2))
    count, logprob = torch.empty(requests, dtype=torch.int32, device=dev), torch.empty(n, dtype=torch.float32, device=dev)
    if requests == 0:
        return Verified(emitted, count, path, logprob)
    nodes = B.int32_array(n_nodes)
    args = B.ts_verify(dev.index, requests, vocab, B.TS_BF16 if logits.dtype == torch.bfloat16 else B.TS_F32, nodes.buffer_info()[0], logits.data_ptr(),
                       logits.stride(0) if n > 1 else vocab, None if draft is None else draft.data_ptr(),
                       vocab if draft is None or n == 1 else draft.stride(0), None if scale is None else scale.data_ptr(),
                       None if draft_scale is None else draft_scale.data_ptr(), tokens.data_ptr(), parents.data_ptr(), u_accept.data_ptr(),
                       u_sample.data_ptr(), emitted.data_ptr(), count.data_ptr(), path.data_ptr(), logprob.data_ptr())
    _check(B.ts_verify_tokens(args, _raw_stream(dev.index)), "ts_verify_tokens")
    return Verified(emitted, count, path, logprob)
