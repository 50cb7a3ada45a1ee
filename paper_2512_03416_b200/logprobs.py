"""Log probabilities of given tokens, with entropy and the best alternatives (ts_token_logprobs). PyTorch supplies
device memory and the stream; all computation happens inside libtokenscale.so.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B
from .decoder import _check, _raw_stream

MAX_GIVEN, MAX_TOP = 8, 32


class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor        # float32 [rows, given]
    rank: torch.Tensor           # int32 [rows, given]: tokens in front of it by (logit descending, index ascending)
    entropy: torch.Tensor        # float32 [rows]
    top_logprob: torch.Tensor    # float32 [rows, n_top]
    top_token: torch.Tensor      # int32 [rows, n_top]


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, n_top: int = 0,
                   scale: Optional[torch.Tensor] = None) -> TokenLogprobs:
    """logits: bf16 or float32 CUDA tensor [rows, vocab], columns next to each other. tokens: int32 [rows, given] (up to 8 per
    row), or [rows]. scale: float32 [rows], inverse temperatures. n_top: up to 32."""
    if not logits.is_cuda or logits.dim() != 2 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be a bf16 or float32 CUDA tensor [rows, vocab]")
    rows, vocab = logits.shape
    if vocab < 1 or (vocab > 1 and logits.stride(1) != 1) or (rows > 1 and logits.stride(0) < vocab):
        raise ValueError("the logits of a row must lie next to each other, and rows may not overlap")
    dev = logits.device
    given = 0
    if tokens is not None:
        tokens = tokens.unsqueeze(1) if tokens.dim() == 1 else tokens
        if tokens.dtype != torch.int32 or tokens.device != dev or tokens.dim() != 2 or tokens.shape[0] != rows or not tokens.is_contiguous():
            raise ValueError(f"tokens must be a contiguous int32 tensor [{rows}, given] on {dev}")
        given = tokens.shape[1]
    if given > MAX_GIVEN or not 0 <= n_top <= MAX_TOP:
        raise ValueError(f"at most {MAX_GIVEN} given tokens and {MAX_TOP} alternatives per row")
    if scale is not None and (scale.dtype != torch.float32 or scale.device != dev or scale.numel() != rows or not scale.is_contiguous()):
        raise ValueError(f"scale must be a contiguous float32 tensor of {rows} values on {dev}")
    # one allocation for each: a slice of a common one costs the host more
    lp, ent, top_lp = (torch.empty(n, dtype=torch.float32, device=dev) for n in ((rows, given), rows, (rows, n_top)))
    rank, top = (torch.empty((rows, n), dtype=torch.int32, device=dev) for n in (given, n_top))
    args = B.ts_logprobs(dev.index, rows, vocab, B.TS_BF16 if logits.dtype == torch.bfloat16 else B.TS_F32, logits.data_ptr(),
                         logits.stride(0) if rows > 1 else vocab, None if scale is None else scale.data_ptr(),
                         None if given == 0 else tokens.data_ptr(), given, n_top, lp.data_ptr(), rank.data_ptr(), ent.data_ptr(),
                         top_lp.data_ptr(), top.data_ptr())
    _check(B.ts_token_logprobs(args, _raw_stream(dev.index)), "ts_token_logprobs")
    return TokenLogprobs(lp, rank, ent, top_lp, top)
