"""Binding of the language-model operators (include/gem_lm.h): the gated linear recurrence,
the distillation loss and the log probabilities of tokens.

Argument marshalling only: tensors are checked for type, layout and size, and their addresses
go to the CUDA library.  Outputs are the caller's tensors.  ``stream`` is a torch stream or a
raw address; the default is torch's current stream.
"""
from __future__ import annotations

import torch

from ._lib import GemSeq, check, lib

GEM_F32, GEM_BF16, GEM_F16 = 0, 1, 2
GEM_GLR_LERP, GEM_GLR_ADD = 0, 1
GEM_GLR_CHUNK = 16
GEM_TOP_MAX = 256

_DTYPES = {torch.float32: GEM_F32, torch.bfloat16: GEM_BF16, torch.float16: GEM_F16}
_F32, _I32, _U8 = torch.float32, torch.int32, torch.uint8

# The current stream's address; where torch offers it without building a Stream object (3 us), that way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(device.index)
        stream = torch.cuda.current_stream(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _dtype(t, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None or not t.is_cuda:
        raise TypeError(f"{what}: expected a float32, bfloat16 or float16 CUDA tensor")
    return d


def _dense(t, what: str, dtype, shape) -> int:
    """Address of a contiguous CUDA tensor of this type and shape."""
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{what}: expected a contiguous {dtype} CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{what}: expected the shape {shape}, got {tuple(t.shape)}")
    return t.data_ptr()


def _seq(t, what: str, like):
    """gem_seq_t of a [B, T, D] tensor of like's type and shape."""
    if t.dtype is not like.dtype or not t.is_cuda:
        raise TypeError(f"{what}: expected a {like.dtype} CUDA tensor")
    if t.shape != like.shape:
        raise ValueError(f"{what}: expected the shape {tuple(like.shape)}, got {tuple(t.shape)}")
    sb, st, sd = t.stride()
    if sd != 1 and t.shape[2] > 1:
        raise TypeError(f"{what}: the channels must be contiguous")
    return GemSeq(t.data_ptr(), sb, st)


def _rows(t, what: str):
    """N, V and the row pitch of a [N, V] tensor with contiguous rows."""
    if t.dim() != 2:
        raise ValueError(f"{what}: expected a [N, V] tensor")
    (N, V), (ld, one) = t.shape, t.stride()
    if one != 1 and V > 1:
        raise TypeError(f"{what}: the rows must be contiguous")
    return N, V, ld if N > 1 or ld > V else V


def _grad_rows(grad, logits) -> int:
    if grad.dtype is not logits.dtype or not grad.is_cuda:
        raise TypeError(f"grad: expected a {logits.dtype} CUDA tensor")
    if grad.shape != logits.shape:
        raise ValueError(f"grad: expected the shape {tuple(logits.shape)}, got {tuple(grad.shape)}")
    return _rows(grad, "grad")[2]


def gem_glr_saved_count(B: int, T: int, D: int) -> int:
    return int(lib().gem_glr_saved_count(B, T, D))


def _reset(t, B, T) -> int:
    return _dense(t.view(torch.uint8) if t.dtype is torch.bool else t, "reset", _U8, (B, T))


def _saved(t, B, T, D):
    return _dense(t, "saved", _F32, (B, -(-T // GEM_GLR_CHUNK), D))


def gem_glr_forward(x, f, h, *, form: int = GEM_GLR_LERP, h0=None, lengths=None, reset=None,
                    h_last=None, saved=None, stream=None) -> None:
    """x, f, h [B, T, D] (channels contiguous, any batch and time strides); h0, h_last [B, D]
    float32; lengths [B] int32; reset [B, T] uint8 or bool; saved [B, ceil(T / 16), D] float32."""
    if x.dim() != 3:
        raise ValueError("x: expected a [B, T, D] tensor")
    B, T, D = x.shape
    check(lib().gem_glr_forward(
        _dtype(x, "x"), form, B, T, D, _seq(x, "x", x), _seq(f, "f", x),
        0 if h0 is None else _dense(h0, "h0", _F32, (B, D)), 0 if lengths is None else _dense(lengths, "lengths", _I32, (B,)),
        0 if reset is None else _reset(reset, B, T), _seq(h, "h", x),
        0 if h_last is None else _dense(h_last, "h_last", _F32, (B, D)), 0 if saved is None else _saved(saved, B, T, D),
        _stream(stream, x.device)), "gem_glr_forward")


def gem_glr_backward(x, f, saved, dh, dx, df, *, form: int = GEM_GLR_LERP, lengths=None,
                     reset=None, dh_last=None, dh0=None, stream=None) -> None:
    """Gradients dx, df [B, T, D] and dh0 [B, D] from dh [B, T, D] and dh_last [B, D]; saved is
    what the forward call saved."""
    if x.dim() != 3:
        raise ValueError("x: expected a [B, T, D] tensor")
    B, T, D = x.shape
    check(lib().gem_glr_backward(
        _dtype(x, "x"), form, B, T, D, _seq(x, "x", x), _seq(f, "f", x),
        0 if lengths is None else _dense(lengths, "lengths", _I32, (B,)), 0 if reset is None else _reset(reset, B, T),
        _saved(saved, B, T, D), _seq(dh, "dh", x),
        0 if dh_last is None else _dense(dh_last, "dh_last", _F32, (B, D)), _seq(dx, "dx", x), _seq(df, "df", x),
        0 if dh0 is None else _dense(dh0, "dh0", _F32, (B, D)), _stream(stream, x.device)), "gem_glr_backward")


def gem_distill(logits, top_idx, top_logits, loss, grad=None, *, teacher_lse=None, labels=None,
                row_scale=None, temperature: float = 1.0, alpha: float = 0.0, stream=None) -> None:
    """logits and grad [N, V] (rows contiguous; grad may be logits or None); top_idx [N, K]
    int32 and top_logits [N, K] float32; loss, teacher_lse, row_scale [N] float32; labels [N]
    int32."""
    N, V, ld = _rows(logits, "logits")
    K = top_idx.shape[1]
    check(lib().gem_distill(
        _dtype(logits, "logits"), N, V, logits.data_ptr(), ld, K,
        _dense(top_idx, "top_idx", _I32, (N, K)), _dense(top_logits, "top_logits", _F32, (N, K)),
        0 if teacher_lse is None else _dense(teacher_lse, "teacher_lse", _F32, (N,)),
        0 if labels is None else _dense(labels, "labels", _I32, (N,)),
        0 if row_scale is None else _dense(row_scale, "row_scale", _F32, (N,)), temperature, alpha,
        _dense(loss, "loss", _F32, (N,)), 0 if grad is None else grad.data_ptr(),
        V if grad is None else _grad_rows(grad, logits), _stream(stream, logits.device)), "gem_distill")


def gem_token_logp(logits, tokens=None, logp=None, entropy=None, *, temperature: float = 1.0,
                   lse=None, top_idx=None, top_logp=None, stream=None) -> None:
    """logits [N, V] (rows contiguous); tokens [N] int32; logp, entropy, lse [N] float32;
    top_idx [N, K] int32 and top_logp [N, K] float32 (both or neither)."""
    N, V, ld = _rows(logits, "logits")
    if (top_idx is None) != (top_logp is None):
        raise ValueError("top_idx and top_logp come together")
    K = 0 if top_idx is None else top_idx.shape[1]
    check(lib().gem_token_logp(
        _dtype(logits, "logits"), N, V, logits.data_ptr(), ld,
        0 if tokens is None else _dense(tokens, "tokens", _I32, (N,)), temperature, K,
        0 if logp is None else _dense(logp, "logp", _F32, (N,)), 0 if entropy is None else _dense(entropy, "entropy", _F32, (N,)),
        0 if lse is None else _dense(lse, "lse", _F32, (N,)), 0 if top_idx is None else _dense(top_idx, "top_idx", _I32, (N, K)),
        0 if top_logp is None else _dense(top_logp, "top_logp", _F32, (N, K)), _stream(stream, logits.device)), "gem_token_logp")


def gem_token_logp_grad(logits, tokens, lse, entropy, dlogp, dentropy, grad, *,
                        temperature: float = 1.0, stream=None) -> None:
    """grad [N, V] (may be logits) from dlogp, dentropy [N] float32 (either may be None) with
    lse and entropy [N] as gem_token_logp wrote them."""
    N, V, ld = _rows(logits, "logits")
    check(lib().gem_token_logp_grad(
        _dtype(logits, "logits"), N, V, logits.data_ptr(), ld,
        0 if tokens is None else _dense(tokens, "tokens", _I32, (N,)), temperature,
        0 if lse is None else _dense(lse, "lse", _F32, (N,)), 0 if entropy is None else _dense(entropy, "entropy", _F32, (N,)),
        0 if dlogp is None else _dense(dlogp, "dlogp", _F32, (N,)),
        0 if dentropy is None else _dense(dentropy, "dentropy", _F32, (N,)), grad.data_ptr(),
        _grad_rows(grad, logits), _stream(stream, logits.device)), "gem_token_logp_grad")
