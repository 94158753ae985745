"""Binding of the language-model operators (include/gem_lm.h): embedding, short causal convolution,
selective state space scan, gated linear recurrence, the distillation and the policy loss, and the log
probabilities of tokens.

Argument marshalling only: tensors are checked for type, layout and size, and their addresses
go to the CUDA library.  Outputs are the caller's tensors.  ``stream`` is a torch stream or a
raw address; the default is torch's current stream.
"""
from __future__ import annotations

import torch

from ._lib import GemSeq, check, lib, pack_seq, pack_ssm, pack_ssm_grad

GEM_F32, GEM_BF16, GEM_F16 = 0, 1, 2
GEM_GLR_LERP, GEM_GLR_ADD = 0, 1
GEM_GLR_CHUNK = 16
GEM_TOP_MAX = 256
GEM_CONV_LINEAR, GEM_CONV_SILU = 0, 1
GEM_SSM_STATES, GEM_SSM_CHUNK = 64, 16

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


def gem_policy(logits, tokens, old_logp, advantage, loss, grad=None, *, ref_logp=None, row_scale=None,
               temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0,
               bonus: float = 0.0, logp=None, entropy=None, stream=None) -> None:
    """logits and grad [N, V] (rows contiguous; grad may be logits or None); tokens [N] int32; old_logp,
    advantage, ref_logp, row_scale, loss, logp, entropy [N] float32."""
    N, V, ld = _rows(logits, "logits")
    check(lib().gem_policy(
        _dtype(logits, "logits"), N, V, logits.data_ptr(), ld, _dense(tokens, "tokens", _I32, (N,)),
        _dense(old_logp, "old_logp", _F32, (N,)), _dense(advantage, "advantage", _F32, (N,)),
        0 if ref_logp is None else _dense(ref_logp, "ref_logp", _F32, (N,)),
        0 if row_scale is None else _dense(row_scale, "row_scale", _F32, (N,)), temperature, clip_low, clip_high, kl, bonus,
        _dense(loss, "loss", _F32, (N,)), 0 if logp is None else _dense(logp, "logp", _F32, (N,)),
        0 if entropy is None else _dense(entropy, "entropy", _F32, (N,)), 0 if grad is None else grad.data_ptr(),
        V if grad is None else _grad_rows(grad, logits), _stream(stream, logits.device)), "gem_policy")


def _matrix(t, what: str, shape):
    """Address and row pitch of a matrix with contiguous rows."""
    if t.shape != shape:
        raise ValueError(f"{what}: expected the shape {shape}, got {tuple(t.shape)}")
    N, D, ld = _rows(t, what)
    return t.data_ptr(), ld


def gem_embed(table, tokens, out, *, scale: float = 1.0, stream=None) -> None:
    """out [N, D] = scale table[tokens] from table [V, D] (rows contiguous, any two types); tokens [N]
    int32."""
    V, D, ld = _rows(table, "table")
    N = tokens.shape[0]
    data, out_ld = _matrix(out, "out", (N, D))
    check(lib().gem_embed(_dtype(table, "table"), _dtype(out, "out"), N, V, D, table.data_ptr(), ld,
                          _dense(tokens, "tokens", _I32, (N,)), scale, data, out_ld, _stream(stream, table.device)), "gem_embed")


def gem_embed_workspace(N: int, V: int, D: int) -> int:
    return int(lib().gem_embed_workspace(N, V, D))


def _space(t, what: str, size: int, dtype) -> int:
    """Address of a workspace of at least this many elements (None where it takes none)."""
    if t is None:
        if size > 0:
            raise ValueError(f"{what}: expected {size} elements")
        return 0
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{what}: expected a contiguous {dtype} CUDA tensor")
    if t.numel() < size:
        raise ValueError(f"{what}: expected {size} elements, got {t.numel()}")
    return t.data_ptr()


def gem_embed_grad(dout, tokens, dtable, workspace, *, scale: float = 1.0, accumulate: bool = False,
                   stream=None) -> None:
    """dtable [V, D] (written, or with accumulate added to) from dout [N, D] (rows contiguous, any two
    types); tokens [N] int32; workspace uint8, gem_embed_workspace(N, V, D) of it."""
    V, D, ld = _rows(dtable, "dtable")
    N = tokens.shape[0]
    data, dout_ld = _matrix(dout, "dout", (N, D))
    check(lib().gem_embed_grad(
        _dtype(dout, "dout"), _dtype(dtable, "dtable"), N, V, D, data, dout_ld, _dense(tokens, "tokens", _I32, (N,)), scale,
        int(accumulate), dtable.data_ptr(), ld, _space(workspace, "workspace", gem_embed_workspace(N, V, D), _U8),
        _stream(stream, dout.device)), "gem_embed_grad")


def _place(t, what: str, like):
    """Address, batch and time stride of a [B, T, D] tensor of like's type and shape (None: of no tensor)."""
    if t is None:
        return 0, 0, 0
    if t.dtype is not like.dtype or not t.is_cuda:
        raise TypeError(f"{what}: expected a {like.dtype} CUDA tensor")
    if t.shape != like.shape:
        raise ValueError(f"{what}: expected the shape {tuple(like.shape)}, got {tuple(t.shape)}")
    sb, st, sd = t.stride()
    if sd != 1 and t.shape[2] > 1:
        raise TypeError(f"{what}: the channels must be contiguous")
    return t.data_ptr(), sb, st


def gem_conv_forward(x, weight, y, *, form: int = GEM_CONV_SILU, bias=None, state=None, lengths=None, reset=None,
                     state_last=None, stream=None) -> None:
    """x, y [B, T, D] (channels contiguous, any batch and time strides); weight [D, W], bias [D], state and
    state_last [B, W - 1, D] float32; lengths [B] int32; reset [B, T] uint8 or bool."""
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x, weight: expected [B, T, D] and [D, W] tensors")
    B, T, D = x.shape
    W = weight.shape[1]
    check(lib().gem_conv_forward(
        _dtype(x, "x"), form, B, T, D, W, pack_seq(*_place(x, "x", x)), _dense(weight, "weight", _F32, (D, W)),
        0 if bias is None else _dense(bias, "bias", _F32, (D,)), 0 if state is None else _dense(state, "state", _F32, (B, W - 1, D)),
        0 if lengths is None else _dense(lengths, "lengths", _I32, (B,)), 0 if reset is None else _reset(reset, B, T),
        pack_seq(*_place(y, "y", x)), 0 if state_last is None else _dense(state_last, "state_last", _F32, (B, W - 1, D)),
        _stream(stream, x.device)), "gem_conv_forward")


def gem_conv_workspace(B: int, T: int, D: int, W: int) -> int:
    return int(lib().gem_conv_workspace(B, T, D, W))


def gem_conv_backward(x, weight, dy, dx, dweight, workspace, *, form: int = GEM_CONV_SILU, bias=None, dbias=None, state=None,
                      lengths=None, reset=None, dstate_last=None, dstate=None, stream=None) -> None:
    """dx [B, T, D], dweight [D, W], dbias [D] and dstate [B, W - 1, D] (the last three may be None) from dy
    [B, T, D] and dstate_last [B, W - 1, D]; workspace float32, gem_conv_workspace(B, T, D, W) of it."""
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x, weight: expected [B, T, D] and [D, W] tensors")
    B, T, D = x.shape
    W = weight.shape[1]
    size = gem_conv_workspace(B, T, D, W) if dweight is not None or dbias is not None else 0
    check(lib().gem_conv_backward(
        _dtype(x, "x"), form, B, T, D, W, pack_seq(*_place(x, "x", x)), _dense(weight, "weight", _F32, (D, W)),
        0 if bias is None else _dense(bias, "bias", _F32, (D,)), 0 if state is None else _dense(state, "state", _F32, (B, W - 1, D)),
        0 if lengths is None else _dense(lengths, "lengths", _I32, (B,)), 0 if reset is None else _reset(reset, B, T),
        pack_seq(*_place(dy, "dy", x)), 0 if dstate_last is None else _dense(dstate_last, "dstate_last", _F32, (B, W - 1, D)),
        pack_seq(*_place(dx, "dx", x)), 0 if dweight is None else _dense(dweight, "dweight", _F32, (D, W)),
        0 if dbias is None else _dense(dbias, "dbias", _F32, (D,)), 0 if dstate is None else _dense(dstate, "dstate", _F32, (B, W - 1, D)),
        _space(workspace, "workspace", size, _F32), _stream(stream, x.device)), "gem_conv_backward")


def _states(t, what: str, like, shape):
    """The same of a [B, T, G, N] tensor of like's type, whose last two dimensions lie side by side."""
    if t.dtype is not like.dtype or not t.is_cuda:
        raise TypeError(f"{what}: expected a {like.dtype} CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{what}: expected the shape {tuple(shape)}, got {tuple(t.shape)}")
    sb, st, sg, sn = t.stride()
    if (sn != 1 and shape[3] > 1) or (sg != shape[3] and shape[2] > 1):
        raise TypeError(f"{what}: groups and states must be contiguous")
    return t.data_ptr(), sb, st


def _ssm(x, dt, A, b, c, z, skip, dt_bias, softplus, lengths, reset):
    """The sizes, and gem_ssm_t."""
    if x.dim() != 3 or b.dim() != 4:
        raise ValueError("x, b: expected [B, T, D] and [B, T, G, N] tensors")
    (B, T, D), (G, N) = x.shape, b.shape[2:]
    shape = (B, T, G, N)
    return B, T, D, N, G, pack_ssm(
        B, T, D, N, G, bool(softplus), *_place(x, "x", x), *_place(dt, "dt", x), *_states(b, "b", x, shape), *_states(c, "c", x, shape),
        *_place(z, "z", x), _dense(A, "A", _F32, (D, N)), 0 if skip is None else _dense(skip, "skip", _F32, (D,)),
        0 if dt_bias is None else _dense(dt_bias, "dt_bias", _F32, (D,)),
        0 if lengths is None else _dense(lengths, "lengths", _I32, (B,)), 0 if reset is None else _reset(reset, B, T))


def gem_ssm_saved_count(B: int, T: int, D: int, N: int) -> int:
    return int(lib().gem_ssm_saved_count(B, T, D, N))


def gem_ssm_workspace(B: int, T: int, D: int, N: int, G: int = 1, *, backward: bool = False) -> int:
    return int(lib().gem_ssm_workspace(B, T, D, N, G, int(backward)))


def gem_ssm_forward(x, dt, A, b, c, y, *, z=None, skip=None, dt_bias=None, softplus: bool = True, h0=None, lengths=None,
                    reset=None, h_last=None, saved=None, workspace=None, stream=None) -> None:
    """x, dt, z, y [B, T, D] (channels contiguous, any batch and time strides); b, c [B, T, G, N] (the last two
    dimensions contiguous); A [D, N], skip, dt_bias [D], h0, h_last [B, D, N], saved [B, ceil(T / 16), D, N]
    float32; lengths [B] int32; reset [B, T] uint8 or bool; workspace float32, gem_ssm_workspace(B, T, D, N, G)
    of it (one step takes none)."""
    B, T, D, N, G, p = _ssm(x, dt, A, b, c, z, skip, dt_bias, softplus, lengths, reset)
    state = (B, D, N)
    check(lib().gem_ssm_forward(
        _dtype(x, "x"), p, 0 if h0 is None else _dense(h0, "h0", _F32, state), pack_seq(*_place(y, "y", x)),
        0 if h_last is None else _dense(h_last, "h_last", _F32, state),
        0 if saved is None else _dense(saved, "saved", _F32, (B, -(-T // GEM_SSM_CHUNK), D, N)),
        _space(workspace, "workspace", 0 if T == 1 else lib().gem_ssm_workspace(B, T, D, N, G, 0), _F32), _stream(stream, x.device)),
        "gem_ssm_forward")


def gem_ssm_backward(x, dt, A, b, c, saved, dy, dx, ddt, dA, db, dc, *, z=None, dz=None, skip=None, dskip=None, dt_bias=None,
                     ddt_bias=None, softplus: bool = True, lengths=None, reset=None, dh_last=None, dh0=None, workspace=None,
                     stream=None) -> None:
    """Gradients of what gem_ssm_forward takes from dy [B, T, D] and dh_last [B, D, N]; saved is what the
    forward call saved; dA, dskip, ddt_bias and dh0 may be None; workspace float32,
    gem_ssm_workspace(B, T, D, N, G, backward=True) of it."""
    B, T, D, N, G, p = _ssm(x, dt, A, b, c, z, skip, dt_bias, softplus, lengths, reset)
    if (z is None) != (dz is None):
        raise ValueError("z and dz come together")
    shape, state = (B, T, G, N), (B, D, N)
    out = pack_ssm_grad(
        *_place(dx, "dx", x), *_place(ddt, "ddt", x), *_states(db, "db", x, shape), *_states(dc, "dc", x, shape), *_place(dz, "dz", x),
        0 if dA is None else _dense(dA, "dA", _F32, (D, N)), 0 if dskip is None else _dense(dskip, "dskip", _F32, (D,)),
        0 if ddt_bias is None else _dense(ddt_bias, "ddt_bias", _F32, (D,)), 0 if dh0 is None else _dense(dh0, "dh0", _F32, state))
    check(lib().gem_ssm_backward(
        _dtype(x, "x"), p, _dense(saved, "saved", _F32, (B, -(-T // GEM_SSM_CHUNK), D, N)), pack_seq(*_place(dy, "dy", x)),
        0 if dh_last is None else _dense(dh_last, "dh_last", _F32, state), out,
        _space(workspace, "workspace", lib().gem_ssm_workspace(B, T, D, N, G, 1), _F32), _stream(stream, x.device)), "gem_ssm_backward")
