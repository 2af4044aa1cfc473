"""What rows of logits say about tokens: log probabilities, entropy, the best alternatives (ouro_token_logprobs of include/ouro.h); and rules on which
tokens may come: penalties, biases, grammar masks (ouro_constrain_logits)."""
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


def allowed_words(mask: torch.Tensor) -> torch.Tensor:
    """A mask [.., vocab] of truth values (True: may come) as the words [.., ceil(vocab / 32)] int32 that ``constrain_logits`` takes."""
    bits = torch.nn.functional.pad(mask.bool(), (0, -mask.shape[-1] % 32)).unflatten(-1, (-1, 32))
    words = (bits.long() << torch.arange(32, device=mask.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def _of_rows(t, name, dtype, rows, width, index):
    """Distance between the rows of an argument [rows, width], 0 for one row for all [width]."""
    shape = t.shape
    if len(shape) == 1:
        shape = (rows, *shape)
    if t.dtype is not dtype or t.get_device() != index or shape != (rows, width) or (width > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: [rows, {width}] of {dtype} on cuda:{index}, with dense rows, is needed (or one row for all, where that is allowed)")
    return t.stride(0) if t.dim() == 2 else 0


def _of_row(t, name, dtype, rows, index):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.dim() != 1 or t.numel() != rows or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous tensor of {rows} elements of {dtype} on cuda:{index} is needed")
    return t.data_ptr()


def constrain_logits(logits: torch.Tensor, *, tokens: torch.Tensor | None = None, lens: torch.Tensor | None = None, repetition: torch.Tensor | None = None,
                     presence: torch.Tensor | None = None, frequency: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                     allowed: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """logits [rows, vocab], f32 or bf16, rows at any distance.  A token that is c > 0 times among the first lens [rows] (None: all) of the row's ``tokens``
    [rows, width] int32 is divided (above 0) or multiplied by ``repetition`` and lowered by ``frequency`` * c + ``presence`` ([rows] f32 each); ``bias`` [vocab] or
    [rows, vocab] f32 is added; what ``allowed`` ([words] or [rows, words] int32, see ``allowed_words``) does not allow becomes -inf.  All penalties count the same tokens
    (to count others for ``repetition`` than for the rest, call twice).  ``out`` may be logits.
    Enqueued on torch's current stream."""
    dtype, index = _DTYPES.get(logits.dtype), logits.get_device()
    if logits.dim() != 2 or dtype is None or index < 0:
        raise ValueError("logits: a CUDA tensor [rows, vocab], f32 or bf16, is needed (this library has no CPU path)")
    rows, vocab = logits.shape
    stride = out_stride = vocab
    contiguous = logits.is_contiguous()
    if not contiguous:
        stride, step = logits.stride()
        if vocab > 1 and step != 1:
            raise ValueError("logits: dense rows are needed")
    if out is None:
        out = torch.empty_like(logits) if contiguous else torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    elif out is logits:
        out_stride = stride
    else:
        if out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != index or (vocab > 1 and out.stride(1) != 1):
            raise ValueError("out has to be like logits")
        out_stride = out.stride(0)
    bias_p = allowed_p = token_p = lens_p = repetition_p = presence_p = frequency_p = None
    bias_stride = allowed_stride = token_stride = width = 0
    if bias is not None:
        bias_stride, bias_p = _of_rows(bias, "bias", torch.float32, rows, vocab, index), bias.data_ptr()
    if allowed is not None:
        allowed_stride, allowed_p = _of_rows(allowed, "allowed", torch.int32, rows, (vocab + 31) // 32, index), allowed.data_ptr()
    if tokens is not None:
        if tokens.dim() != 2:
            raise ValueError("tokens: [rows, width] of torch.int32 is needed")
        width = tokens.shape[1]
        token_stride = _of_rows(tokens, "tokens", torch.int32, rows, width, index)
        lens_p, repetition_p = _of_row(lens, "lens", torch.int32, rows, index), _of_row(repetition, "repetition", torch.float32, rows, index)
        presence_p, frequency_p = _of_row(presence, "presence", torch.float32, rows, index), _of_row(frequency, "frequency", torch.float32, rows, index)
        if width > 0:
            token_p = tokens.data_ptr()
        else:                                                      # nothing has been said
            lens_p = repetition_p = presence_p = frequency_p = None
    elif lens is not None or repetition is not None or presence is not None or frequency is not None:
        raise ValueError("lens, repetition, presence and frequency come with tokens")
    _check(lib().ouro_constrain_logits(logits.data_ptr(), dtype, stride, rows, vocab, token_p, token_stride, width, lens_p, repetition_p, presence_p, frequency_p,
                                       bias_p, bias_stride, allowed_p, allowed_stride, out.data_ptr(), out_stride, current_stream(index)))
    return out
