"""What rows of logits say about tokens: log probabilities, entropy, the best alternatives (ouro_token_logprobs of include/ouro.h)."""
from __future__ import annotations

from typing import NamedTuple

import torch

from .binding import OURO_BF16, OURO_F32, _check, current_stream, lib

_DTYPES = {torch.float32: OURO_F32, torch.bfloat16: OURO_BF16}


class TokenScores(NamedTuple):
    logprob: torch.Tensor | None        # [rows] f32: of the given tokens
    entropy: torch.Tensor               # [rows] f32, in nats
    top_ids: torch.Tensor | None        # [rows, n_top] int32: best first, ties by the lowest id
    top_logprobs: torch.Tensor | None   # [rows, n_top] f32


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, n_top: int = 0) -> TokenScores:
    """logits [rows, vocab], f32 or bf16, rows at any distance; tokens [rows] int32 (None: no token is asked about); n_top <= 32.
    Enqueued on torch's current stream."""
    if logits.dim() != 2 or logits.dtype not in _DTYPES or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits: a CUDA tensor [rows, vocab], f32 or bf16, with dense rows is needed (this library has no CPU path)")
    rows, vocab = logits.shape
    dev = logits.device
    if tokens is not None and (tokens.dtype is not torch.int32 or tokens.device != dev or tokens.numel() != rows or not tokens.is_contiguous()):
        raise ValueError(f"tokens: a contiguous int32 tensor of {rows} elements on {dev} is needed")
    entropy = torch.empty(rows, dtype=torch.float32, device=dev)
    logprob = torch.empty_like(entropy) if tokens is not None else None
    ids = torch.empty_strided((rows, n_top), (n_top, 1), dtype=torch.int32, device=dev) if n_top > 0 else None
    top = torch.empty_like(ids, dtype=torch.float32) if n_top > 0 else None
    _check(lib().ouro_token_logprobs(logits.data_ptr(), _DTYPES[logits.dtype], logits.stride(0), rows, vocab,
                                     None if tokens is None else tokens.data_ptr(), n_top, None if tokens is None else logprob.data_ptr(), entropy.data_ptr(),
                                     None if ids is None else ids.data_ptr(), None if top is None else top.data_ptr(), current_stream(dev.index)))
    return TokenScores(logprob, entropy, ids, top)
