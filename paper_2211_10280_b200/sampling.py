"""The draw of the next token from logits, over torch CUDA tensors."""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as B
from .layers import _device_of
from .operators import _FLOATS, _current_stream, _need, _written

_at = C.byref


_INFINITY = float("inf")


def _setting(name, x, dtype, n, index):
    if not isinstance(x, torch.Tensor):
        return None, x
    if x.shape != (n,) or x.dtype != dtype or x.get_device() != index or not x.is_contiguous():
        raise ValueError(f"{name}: a number, or contiguous {dtype} of ({n},) on the logits' device")
    return x.data_ptr(), 0


def sample(logits, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, logprobs: bool = False):
    """Draws a token for each row of logits (n, V), with the random numbers `uniform` (float32 (n,), in [0, 1)).

    Tokens in the order of (logit descending, id ascending) are kept if they are among the first top_k (0: all), of those the ones
    with less than top_p of the weight before them, and of those the ones whose probability is at least min_p times the largest; the
    token is the lowest id whose running kept weight, ids ascending, exceeds uniform times the whole, weights being exp((logit -
    largest) / temperature).  temperature 0: the lowest id of the largest logit.  Each setting is a number, or a tensor with one for
    each row (float32; top_k int32) in which a value <= 0 (top_p: >= 1) switches that setting off (temperature: draws the largest).

    A logit of minus infinity, or NaN, is never drawn; a row without any other has token -1.  Returns int64 (n,) (`out`, if
    given), with logprobs also the logarithms, float32, of the tokens' probabilities among those kept.  Neither takes part in autograd."""
    index = _device_of(logits, "logits")
    kind = _FLOATS.get(logits.dtype)
    if kind is None or logits.dim() != 2:
        raise ValueError(f"logits: {tuple(logits.shape)} of {logits.dtype}; (n, V) of float32, bfloat16 or float16 goes")
    n, V = logits.shape
    row, column = logits.stride()
    if (column != 1 and V > 1) or (row < V and n > 1):
        logits = logits.contiguous()
        row = V
    if uniform.shape != (n,) or uniform.dtype != torch.float32 or uniform.get_device() != index or not uniform.is_contiguous():
        raise ValueError(f"uniform: contiguous float32 of ({n},) on the logits' device")
    # each setting: (address of one for each row, or None; the one for all)
    ts, t = (None, temperature) if temperature.__class__ is float else _setting("temperature", temperature, torch.float32, n, index)
    ks, k = (None, top_k) if top_k.__class__ is int else _setting("top_k", top_k, torch.int32, n, index)
    ps, p = (None, top_p) if top_p.__class__ is float else _setting("top_p", top_p, torch.float32, n, index)
    ms, m = (None, min_p) if min_p.__class__ is float else _setting("min_p", min_p, torch.float32, n, index)
    if not (0 <= t < _INFINITY and 0 <= k < 1 << 31 and p >= 0 and 0 <= m <= 1):
        raise ValueError(f"temperature {t}, top_k {k}, top_p {p} or min_p {m} is out of range")
    given = out
    if out is None:
        out = torch.empty(n, dtype=torch.int64, device=logits.device)
    elif out.shape != (n,) or out.dtype != torch.int64 or out.get_device() != index or not out.is_contiguous():
        raise ValueError(f"out: contiguous int64 of ({n},) on the logits' device")
    logprob = torch.empty_like(uniform) if logprobs else None
    h = B.Draw(uniform.data_ptr(), out.data_ptr(), None if logprob is None else logprob.data_ptr(), ts, ps, ms, ks, t, p, m, k, n)
    rc = B.lib().tensair_sample(_at(h), _at(B.Rows(logits.data_ptr(), row if n > 1 else V, V, kind)), _current_stream(index))
    if rc:
        B._check(rc, "tensair_sample")
    if given is not None:
        _written(given)
    return (out, logprob) if logprobs else out
