"""Thin ctypes binding of libfpdt_tokenwise.so (include/fpdt_tokenwise.h): argument marshalling
only.  Tensors are torch tensors used as memory handles; there is no fallback."""
import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libfpdt_tokenwise.so")
_lib = None


FPDT_TW_GELU = 0
FPDT_TW_SWIGLU = 1
FPDT_TW_F32, FPDT_TW_BF16 = 0, 1
FPDT_TW_ROPE_HALF, FPDT_TW_ROPE_INTERLEAVED = 0, 1
FPDT_TW_ROPE_PLAIN, FPDT_TW_ROPE_LINEAR, FPDT_TW_ROPE_RAISED, FPDT_TW_ROPE_PARTS = range(4)
FPDT_TW_RMSNORM, FPDT_TW_LAYERNORM = 0, 1
FPDT_TW_ACT_NONE, FPDT_TW_ACT_GELU, FPDT_TW_ACT_SILU = 0, 1, 2
FPDT_TW_JOIN_ADD, FPDT_TW_JOIN_TIMES = 0, 1
FPDT_TW_ADAMW_ZERO_GRAD = 1 << 0
FPDT_TW_STATE_BLOCK = 128  # elements that share an exponent byte of 8-bit states


class FpdtTwError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("fpdt_tw status %d: %s" % (status, text))
        self.status = status


def load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libfpdt_tokenwise.so is not built: run `python -m paper_2408_16978_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, ci, cf, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    L.fpdt_tw_loss_workspace_bytes.restype = sz
    L.fpdt_tw_loss_workspace_bytes.argtypes = [i64, ci, ci, ci]
    L.fpdt_tw_loss_fwd_bwd.restype = ci
    L.fpdt_tw_loss_fwd_bwd.argtypes = [vp, vp, vp, cf, vp, vp, vp, vp, i64, ci, ci, ci, vp, sz, vp]
    L.fpdt_tw_linear_fwd.restype = ci
    L.fpdt_tw_linear_fwd.argtypes = [vp, vp, vp, i64, ci, ci, ci, vp]
    L.fpdt_tw_linear_bwd.restype = ci
    L.fpdt_tw_linear_bwd.argtypes = [vp, vp, vp, vp, vp, i64, ci, ci, ci, vp]
    L.fpdt_tw_ffn_workspace_bytes.restype = sz
    L.fpdt_tw_ffn_workspace_bytes.argtypes = [i64, ci, ci, ci, ci, ci]
    L.fpdt_tw_ffn_fwd.restype = ci
    L.fpdt_tw_ffn_fwd.argtypes = [vp, vp, vp, vp, vp, i64, ci, ci, ci, ci, vp, sz, vp]
    L.fpdt_tw_ffn_bwd.restype = ci
    L.fpdt_tw_ffn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, ci, ci, ci, ci, vp, sz, vp]
    cd, ci64p, cu = ctypes.c_double, [vp, i64], ctypes.c_uint
    rope = ci64p * 6 + [vp, i64, vp, cf, i64, ci, ci, ci, ci, ci, ci, vp]
    L.fpdt_tw_rope_fwd.restype = ci
    L.fpdt_tw_rope_fwd.argtypes = rope
    L.fpdt_tw_rope_bwd.restype = ci
    L.fpdt_tw_rope_bwd.argtypes = rope
    L.fpdt_tw_rope_freqs.restype = ci
    L.fpdt_tw_rope_freqs.argtypes = [ci, cd, ci, cd, cd, cd, cd, vp]
    L.fpdt_tw_norm_fwd.restype = ci
    L.fpdt_tw_norm_fwd.argtypes = [vp] * 7 + [i64, ci, ci, cf, ci, vp]
    L.fpdt_tw_norm_bwd_workspace_bytes.restype = sz
    L.fpdt_tw_norm_bwd_workspace_bytes.argtypes = [i64, ci, ci]
    L.fpdt_tw_norm_bwd.restype = ci
    L.fpdt_tw_norm_bwd.argtypes = [vp] * 8 + [i64, ci, ci, ci, vp, sz, vp]
    cu64 = ctypes.c_uint64
    for name, args in (("affine_fwd", [vp] * 6 + [i64, ci, ci, ci, ci, vp, sz, vp]), ("affine_bwd", [vp] * 6 + [i64, ci, ci, ci, vp, ci, vp, sz, vp]),
                       ("dropout_fwd", [vp] * 3 + [i64, i64, cd, cu64, i64, vp, ci, vp]), ("dropout_bwd", [vp] * 2 + [i64, i64, cd, cu64, i64, vp, ci, vp]),
                       ("experts_sort", [vp] * 3 + [i64, ci, ci, vp, sz, vp]), ("experts_gather_fwd", [vp] * 3 + [i64, ci, ci, ci, vp]),
                       ("experts_gather_bwd", [vp] * 4 + [i64, ci, ci, ci, vp]), ("experts_combine_fwd", [vp] * 5 + [i64, ci, ci, ci, vp]),
                       ("experts_combine_bwd", [vp] * 6 + [i64, ci, ci, ci, vp]), ("experts_affine_fwd", [vp] * 7 + [i64, ci, ci, ci, ci, ci, vp]),
                       ("experts_linear_bwd", [vp] * 6 + [i64, ci, ci, ci, vp])):
        f = getattr(L, "fpdt_tw_" + name)
        f.restype, f.argtypes = ci, args
    for name, args in (("affine", [i64, ci, ci]), ("affine_bwd", [i64, ci, ci]), ("experts_sort", [i64, ci])):
        f = getattr(L, "fpdt_tw_%s_workspace_bytes" % name)
        f.restype, f.argtypes = sz, args
    L.fpdt_tw_grad_norm_workspace_bytes.restype = sz
    L.fpdt_tw_grad_norm_workspace_bytes.argtypes = [ci]
    L.fpdt_tw_grad_norm.restype = ci
    L.fpdt_tw_grad_norm.argtypes = [vp, ci, ci, cd, vp, vp, sz, vp]
    L.fpdt_tw_adamw_step.restype = ci
    L.fpdt_tw_adamw_step.argtypes = [vp, ci, ci, ci, cd, cd, cd, cd, i64, vp, vp, vp, cu, cu, vp]
    L.fpdt_tw_adamw_unpack.restype = ci
    L.fpdt_tw_adamw_unpack.argtypes = [vp, ci, vp]
    L.fpdt_tw_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def fpdt_tw_last_error() -> str:
    return load().fpdt_tw_last_error().decode()


def fpdt_tw_loss_workspace_bytes(rows, hidden, vocab, n_chunks) -> int:
    return int(load().fpdt_tw_loss_workspace_bytes(rows, hidden, vocab, n_chunks))


def _ptr(t):
    return None if t is None else t.data_ptr()


def fpdt_tw_loss_fwd_bwd(H, W, target, grad_scale, loss, lse, dH, dW, n_chunks, workspace, stream=None):
    """H [rows, hidden] bf16, W [vocab, hidden] bf16, target [rows] int32; loss, lse [rows] fp32;
    dH [rows, hidden] bf16 or None; dW [vocab, hidden] fp32 (accumulated into) or None."""
    rows, hidden = H.shape
    vocab = W.shape[0]
    if stream is None:
        stream = torch.cuda.current_stream()
    st = load().fpdt_tw_loss_fwd_bwd(_ptr(H), _ptr(W), _ptr(target), float(grad_scale), _ptr(loss), _ptr(lse),
                                     _ptr(dH), _ptr(dW), rows, hidden, vocab, n_chunks, _ptr(workspace),
                                     0 if workspace is None else workspace.numel() * workspace.element_size(),
                                     stream.cuda_stream)
    if st != 0:
        raise FpdtTwError(st, fpdt_tw_last_error())


def _check(st):
    if st != 0:
        raise FpdtTwError(st, fpdt_tw_last_error())


def _stream(stream):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def fpdt_tw_linear_fwd(X, W, Y, n_chunks, stream=None):
    """Y [rows, n_out] = X [rows, n_in] W^T, W [n_out, n_in]; all bf16."""
    rows, n_in = X.shape
    _check(load().fpdt_tw_linear_fwd(_ptr(X), _ptr(W), _ptr(Y), rows, n_in, W.shape[0], n_chunks, _stream(stream)))


def fpdt_tw_linear_bwd(X, W, dY, dX, dW, n_chunks, stream=None):
    """dX (bf16, written, or None) = dY W;  dW (fp32, accumulated into, or None) += dY^T X."""
    rows, n_in = X.shape
    _check(load().fpdt_tw_linear_bwd(_ptr(X), _ptr(W), _ptr(dY), _ptr(dX), _ptr(dW), rows, n_in, W.shape[0],
                                     n_chunks, _stream(stream)))


def fpdt_tw_ffn_workspace_bytes(rows, n_model, n_ffn, act, n_chunks, is_bwd) -> int:
    return int(load().fpdt_tw_ffn_workspace_bytes(rows, n_model, n_ffn, act, n_chunks, int(bool(is_bwd))))


def fpdt_tw_ffn_fwd(X, W1, W3, W2, Y, act, n_chunks, workspace, stream=None):
    """X, Y [rows, n_model] bf16; W1, W3 [n_ffn, n_model]; W2 [n_model, n_ffn]; W3 None for GELU."""
    rows, n_model = X.shape
    _check(load().fpdt_tw_ffn_fwd(_ptr(X), _ptr(W1), _ptr(W3), _ptr(W2), _ptr(Y), rows, n_model, W1.shape[0], act,
                                  n_chunks, _ptr(workspace), _nbytes(workspace), _stream(stream)))


def fpdt_tw_ffn_bwd(X, W1, W3, W2, dY, dX, dW1, dW3, dW2, act, n_chunks, workspace, stream=None):
    """dX bf16 (written); dW1, dW3, dW2 fp32 (accumulated into; any may be None)."""
    rows, n_model = X.shape
    _check(load().fpdt_tw_ffn_bwd(_ptr(X), _ptr(W1), _ptr(W3), _ptr(W2), _ptr(dY), _ptr(dX), _ptr(dW1), _ptr(dW3),
                                  _ptr(dW2), rows, n_model, W1.shape[0], act, n_chunks, _ptr(workspace),
                                  _nbytes(workspace), _stream(stream)))


# ---- rotary positions, normalisation, optimizer: shapes, types and places are checked here (the library sees addresses only)
_TYPES = {torch.float32: FPDT_TW_F32, torch.bfloat16: FPDT_TW_BF16}


def _dtype_code(t):
    if t.dtype not in _TYPES:
        raise TypeError("fpdt_tw: tensors must be float32 or bfloat16, got %s" % t.dtype)
    return _TYPES[t.dtype]


def _expect(name, t, shape, dtype, device):
    """`t` is a contiguous tensor of that shape and type on that device (an index)."""
    if t.dtype != dtype or t.get_device() != device:
        raise TypeError("fpdt_tw: %s must be %s on device %s, got %s on %s" % (name, dtype, device, t.dtype, t.device))
    if t.shape != shape or not t.is_contiguous():
        raise ValueError("fpdt_tw: %s must be contiguous and %s, got %s with strides %s" % (name, tuple(shape), tuple(t.shape), t.stride()))
    return t.data_ptr()


# Sizes that the library takes as an int: ctypes would pass the lower 32 bits of larger ones, and with them another shape.
_INT_BITS = 30


def _room(workspace, device):
    """Address and bytes of a workspace (None: none, which the library refuses where it needs one)."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != device:
        raise TypeError("fpdt_tw: the workspace must be on device %s, got %s" % (device, workspace.device))
    if not workspace.is_contiguous():
        raise ValueError("fpdt_tw: the workspace must be contiguous, got %s with strides %s" % (tuple(workspace.shape), workspace.stride()))
    return workspace.data_ptr(), _nbytes(workspace)


def _current(t):
    """The index of `t`'s device, which has to be the current one: calls go to its stream."""
    device = t.get_device()
    if device < 0 or device != torch.cuda.current_device():
        raise ValueError("fpdt_tw: tensors must be on the current device, got %s" % t.device)
    return device


def _raw_stream(stream, device):
    # (a stream object of torch's costs as much to make as the rest of a small call)
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def fpdt_tw_rope_freqs(rot, base, scaling=FPDT_TW_ROPE_PLAIN, factor=1.0, context=0.0, low=1.0, high=4.0):
    """[rot / 2] fp64 on the host: radians per token of each pair.  Copy it to the device once."""
    if rot >> _INT_BITS:
        raise FpdtTwError(1, "rot=%d must be even and in [2, 8192]" % rot)
    out = torch.empty(max(int(rot) // 2, 1), dtype=torch.float64)
    _check(load().fpdt_tw_rope_freqs(rot, base, scaling, factor, context, low, high, out.data_ptr()))
    return out


def _rope(call, ins, outs, freqs, positions, position0, amplitude, layout, stream):
    Q, dtype = ins[0], ins[0].dtype
    device, code = _current(Q), _dtype_code(Q)
    if Q.dim() != 3:
        raise ValueError("fpdt_tw: Q must be [rows, heads, D], got %s" % (tuple(Q.shape),))
    rows, Hq, D = Q.shape
    other = ins[1] if ins[1] is not None else ins[2]
    Hkv = 0 if other is None else other.size(1)
    args = []
    for name, heads, t, o in zip("QKVQKV", (Hq, Hkv, Hkv) * 2, ins + outs, outs + ins):
        if t is None:
            if o is not None:
                raise ValueError("fpdt_tw: %s is given on one side only" % name)
            args += (None, 0)
            continue
        if t.dtype != dtype or t.get_device() != device:
            raise TypeError("fpdt_tw: %s must be %s on device %s, got %s on %s" % (name, dtype, device, t.dtype, t.device))
        strides = t.stride()
        if t.shape != (rows, heads, D) or (D > 1 and strides[2] != 1) or (heads > 1 and strides[1] != D):
            raise ValueError("fpdt_tw: %s must be %s with contiguous heads, got %s with strides %s" % (name, (rows, heads, D), tuple(t.shape), strides))
        args += (t.data_ptr(), strides[0] if rows > 1 else heads * D)
    half = freqs.numel()
    if (Hq | Hkv | D | half) >> _INT_BITS:
        raise FpdtTwError(2, "sizes beyond the launch limits")
    args += (None if positions is None else _expect("positions", positions, (rows,), torch.int64, device), position0,
             _expect("freqs", freqs, (half,), torch.float64, device), amplitude, rows, Hq, Hkv, D, 2 * half, layout, code, _raw_stream(stream, device))
    _check(call(*args))


def fpdt_tw_rope_fwd(Q, K, V, Qo, Ko, Vo, freqs, positions=None, position0=0, amplitude=1.0, layout=FPDT_TW_ROPE_HALF, stream=None):
    """Qo, Ko: the heads of Q [rows, Hq, D] and K [rows, Hkv, D] turned by their tokens' positions; Vo: V copied.  Tokens may be
    any distance apart (slices of a [rows, (Hq + 2 Hkv) D] product).  K and V, or V, may be None on both sides."""
    _rope(load().fpdt_tw_rope_fwd, (Q, K, V), (Qo, Ko, Vo), freqs, positions, position0, amplitude, layout, stream)


def fpdt_tw_rope_bwd(dQo, dKo, dVo, dQ, dK, dV, freqs, positions=None, position0=0, amplitude=1.0, layout=FPDT_TW_ROPE_HALF, stream=None):
    """dQ, dK, dV (slices of the product's gradient, say): the gradients of the forward's inputs."""
    _rope(load().fpdt_tw_rope_bwd, (dQo, dKo, dVo), (dQ, dK, dV), freqs, positions, position0, amplitude, layout, stream)


def fpdt_tw_norm_fwd(X, R, W, B, S, Y, stats, eps, kind=FPDT_TW_RMSNORM, stream=None):
    """S = X + R (R and S, or S, may be None), Y = normalised S times W [hidden] (plus B, LAYERNORM).  stats: None, or fp32 of
    rows (RMSNORM: rstd) or 2 rows (LAYERNORM: mean, rstd) values for the backward."""
    device, dtype, code = _current(X), X.dtype, _dtype_code(X)
    rows, hidden = X.shape
    if hidden >> _INT_BITS:
        raise FpdtTwError(2, "hidden=%d beyond the launch limits" % hidden)
    at = [None if t is None else _expect(name, t, shape, dtype, device) for name, t, shape in (
        ("X", X, X.shape), ("R", R, X.shape), ("W", W, (hidden,)), ("B", B, (hidden,)), ("S", S, X.shape), ("Y", Y, X.shape))]
    _check(load().fpdt_tw_norm_fwd(*at, _stats(stats, rows, kind, device), rows, hidden, kind, eps, code, _raw_stream(stream, device)))


def _stats(stats, rows, kind, device):
    if stats is None:
        return None
    n = rows * (2 if kind == FPDT_TW_LAYERNORM else 1)
    if stats.dtype != torch.float32 or stats.get_device() != device or stats.numel() != n or not stats.is_contiguous():
        raise ValueError("fpdt_tw: stats must be %d contiguous float32 values on device %s" % (n, device))
    return stats.data_ptr()


def fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, kind=FPDT_TW_RMSNORM) -> int:
    return 0 if hidden >> _INT_BITS else int(load().fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, kind))


def fpdt_tw_norm_bwd(S, W, stats, dY, dR, dX, dW, dB, kind=FPDT_TW_RMSNORM, workspace=None, stream=None):
    """dX (written) = gradient through the norm plus dR (or None); dW, dB fp32 [hidden] (accumulated into, or None)."""
    device, dtype, code = _current(S), S.dtype, _dtype_code(S)
    rows, hidden = S.shape
    if hidden >> _INT_BITS:
        raise FpdtTwError(2, "hidden=%d beyond the launch limits" % hidden)
    at = [None if t is None else _expect(name, t, shape, dtype, device) for name, t, shape in (
        ("S", S, S.shape), ("W", W, (hidden,)), ("dY", dY, S.shape), ("dR", dR, S.shape), ("dX", dX, S.shape))]
    sums = [None if t is None else _expect(name, t, (hidden,), torch.float32, device) for name, t in (("dW", dW), ("dB", dB))]
    _check(load().fpdt_tw_norm_bwd(at[0], at[1], _stats(stats, rows, kind, device), *at[2:], *sums, rows, hidden, kind, code, *_room(workspace, device),
                                   _raw_stream(stream, device)))


# ---- products with something behind them, dropout, experts
def _sizes(*sizes):
    for n in sizes:
        if n >> _INT_BITS:
            raise FpdtTwError(2, "sizes beyond the launch limits")


def _half(name, t, shape, device):
    return None if t is None else _expect(name, t, shape, torch.bfloat16, device)


def fpdt_tw_affine_workspace_bytes(rows, n_in, n_out) -> int:
    return 0 if (n_in | n_out) >> _INT_BITS else int(load().fpdt_tw_affine_workspace_bytes(rows, n_in, n_out))


def fpdt_tw_affine_fwd(X, W, B, R, Z, Y, act=FPDT_TW_ACT_NONE, join=FPDT_TW_JOIN_ADD, workspace=None, stream=None):
    """Y [rows, n_out] = act(X W^T + B) plus R (JOIN_ADD; R may be None) or times R (JOIN_TIMES); Z: what the activation is taken of, for the
    backward, or None.  X [rows, n_in], W [n_out, n_in], B [n_out] or None; all bf16.  Y may be R itself."""
    device, (rows, n_in), n_out = _current(X), X.shape, W.size(0)
    _sizes(n_in, n_out)
    out = (rows, n_out)
    _check(load().fpdt_tw_affine_fwd(_half("X", X, X.shape, device), _half("W", W, (n_out, n_in), device), _half("B", B, (n_out,), device), _half("R", R, out, device),
                                     _half("Z", Z, out, device), _half("Y", Y, out, device), rows, n_in, n_out, act, join, *_room(workspace, device),
                                     _raw_stream(stream, device)))


def _experts_of(offsets, device):
    """(address, number of experts) of offsets, int32 [experts + 1]."""
    if offsets is None:
        return None, 1
    if offsets.dim() != 1 or offsets.numel() < 2:
        raise ValueError("fpdt_tw: offsets must be [experts + 1], got %s" % (tuple(offsets.shape),))
    experts = offsets.numel() - 1
    _sizes(experts)
    return _expect("offsets", offsets, offsets.shape, torch.int32, device), experts


def fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, experts=1) -> int:
    return 0 if (n_out | experts) >> _INT_BITS else int(load().fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, experts))


def fpdt_tw_affine_bwd(Z, R, dY, dZ, dR, dB, act=FPDT_TW_ACT_NONE, join=FPDT_TW_JOIN_ADD, offsets=None, workspace=None, stream=None):
    """dZ (written) = dY act'(Z), times R with JOIN_TIMES, where dR (written, or None) = dY act(Z); dB (accumulated into, or None): fp32 [n_out], or
    [experts, n_out] where offsets (of fpdt_tw_experts_sort) say whose rows are whose.  Then fpdt_tw_linear_bwd or fpdt_tw_experts_linear_bwd with dZ
    for dY.  Z, R, dZ are None where they are not needed; dZ and dR may be Z, R or dY themselves."""
    device, (rows, n_out) = _current(dY), dY.shape
    _sizes(n_out)
    place, experts = _experts_of(offsets, device)
    z, r, dy, dz, dr = (_half(name, t, dY.shape, device) for name, t in (("Z", Z), ("R", R), ("dY", dY), ("dZ", dZ), ("dR", dR)))
    db = None if dB is None else _expect("dB", dB, (n_out,) if offsets is None and dB.dim() == 1 else (experts, n_out), torch.float32, device)
    _check(load().fpdt_tw_affine_bwd(z, r, dy, dz, dr, db, rows, n_out, act, join, place, experts, *_room(workspace, device), _raw_stream(stream, device)))


def _dropout(call, tensors, p, seed, step, first, step_dev, stream):
    X = tensors[0][1]
    device, code = _current(X), _dtype_code(X)
    at = [None if t is None else _expect(name, t, X.shape, X.dtype, device) for name, t in tensors]
    if not 0 <= seed < 1 << 64:
        raise ValueError("fpdt_tw: seed must be in [0, 2^64), got %d" % seed)
    if not (-1 << 63 <= step < 1 << 63 and 0 <= first < 1 << 62):
        raise FpdtTwError(2, "step beyond 64 bits, or first beyond [0, 2^62)")
    _check(call(*at, X.numel(), first, p, seed, step, None if step_dev is None else _expect("step_dev", step_dev, step_dev.shape if step_dev.numel() == 1 else (1,), torch.int64, device),
                code, _raw_stream(stream, device)))


def fpdt_tw_dropout_fwd(X, R, Y, p, seed, step=0, first=0, step_dev=None, stream=None):
    """Y = X dropped with probability p (to a 65536th) and scaled, plus R (or None).  The choice depends on seed (a number of its own for each layer),
    step and the element's number, from `first` on: a chunk of a sequence gives its first element's number in the whole.  step_dev: None, or one int64
    on the device in place of step.  Y may be X or R itself."""
    _dropout(load().fpdt_tw_dropout_fwd, (("X", X), ("R", R), ("Y", Y)), p, seed, step, first, step_dev, stream)


def fpdt_tw_dropout_bwd(dY, dX, p, seed, step=0, first=0, step_dev=None, stream=None):
    """dX: dY where the forward of the same seed, step and first kept its element, scaled; 0 elsewhere.  dX may be dY itself."""
    _dropout(load().fpdt_tw_dropout_bwd, (("dY", dY), ("dX", dX)), p, seed, step, first, step_dev, stream)


def fpdt_tw_experts_sort_workspace_bytes(assignments, experts) -> int:
    return 0 if experts >> _INT_BITS else int(load().fpdt_tw_experts_sort_workspace_bytes(assignments, experts))


def fpdt_tw_experts_sort(expert, offsets, place, workspace, stream=None):
    """offsets [experts + 1]: where each expert's rows begin, and all of them end; place [rows, top]: the row of each assignment of expert
    [rows, top], or -1 where that is no expert's number.  All int32.  In the order of experts, then tokens."""
    device, (rows, top) = _current(expert), expert.shape
    _sizes(top)
    at, experts = _experts_of(offsets, device)
    _check(load().fpdt_tw_experts_sort(_expect("expert", expert, expert.shape, torch.int32, device), at, _expect("place", place, expert.shape, torch.int32, device),
                                       rows, top, experts, *_room(workspace, device), _raw_stream(stream, device)))


def _routed(device, place, one, wide, weights=()):
    """Checks of tokens [rows, hidden] (`one`) and their copies [rows top, hidden] (`wide`): addresses of place, of `one`, `wide` and `weights` in that order, and the sizes."""
    if place.dim() != 2:
        raise ValueError("fpdt_tw: place must be [rows, top], got %s" % (tuple(place.shape),))
    (rows, top), some = place.shape, next(t for _, t in one + wide if t is not None)
    hidden, dtype, code = some.size(-1), some.dtype, _dtype_code(some)
    _sizes(top, hidden)
    at = [_expect("place", place, place.shape, torch.int32, device)]
    at += [None if t is None else _expect(name, t, (rows, hidden), dtype, device) for name, t in one]
    at += [None if t is None else _expect(name, t, (rows * top, hidden), dtype, device) for name, t in wide]
    at += [None if t is None else _expect(name, t, (rows, top), torch.float32, device) for name, t in weights]
    return at, (rows, top, hidden, code)


def fpdt_tw_experts_gather_fwd(X, place, Xs, stream=None):
    """Xs [rows top, hidden]: the tokens of X [rows, hidden] at their places; rows without an assignment are left as they were."""
    device = _current(X)
    (p, x, xs), sizes = _routed(device, place, (("X", X),), (("Xs", Xs),))
    _check(load().fpdt_tw_experts_gather_fwd(x, p, xs, *sizes, _raw_stream(stream, device)))


def fpdt_tw_experts_gather_bwd(dXs, place, R, dX, stream=None):
    """dX [rows, hidden]: sums of the gradients dXs [rows top, hidden] over each token's places, plus R (or None; dX may be R itself)."""
    device = _current(dXs)
    (p, r, dx, dxs), sizes = _routed(device, place, (("R", R), ("dX", dX)), (("dXs", dXs),))
    _check(load().fpdt_tw_experts_gather_bwd(dxs, p, r, dx, *sizes, _raw_stream(stream, device)))


def fpdt_tw_experts_combine_fwd(Ys, weight, place, R, Y, stream=None):
    """Y [rows, hidden]: sums of Ys [rows top, hidden] over each token's places, weighted (fp32 [rows, top]), plus R (or None; Y may be R itself)."""
    device = _current(Ys)
    (p, r, y, ys, w), sizes = _routed(device, place, (("R", R), ("Y", Y)), (("Ys", Ys),), (("weight", weight),))
    _check(load().fpdt_tw_experts_combine_fwd(ys, w, p, r, y, *sizes, _raw_stream(stream, device)))


def fpdt_tw_experts_combine_bwd(Ys, weight, place, dY, dYs, dweight, stream=None):
    """dYs (written, or None; rows without an assignment are left as they were): each place's token of dY, weighted; dweight (written, or None): the products
    of dY with each place's row of Ys.  dYs may be Ys itself."""
    device = _current(dY)
    (p, dy, ys, dys, w, dw), sizes = _routed(device, place, (("dY", dY),), (("Ys", Ys), ("dYs", dYs)), (("weight", weight), ("dweight", dweight)))
    _check(load().fpdt_tw_experts_combine_bwd(ys, w, p, dy, dys, dw, *sizes, _raw_stream(stream, device)))


def fpdt_tw_experts_affine_fwd(X, W, B, R, Z, Y, offsets, act=FPDT_TW_ACT_NONE, join=FPDT_TW_JOIN_ADD, stream=None):
    """fpdt_tw_affine_fwd for the rows of each expert (offsets of fpdt_tw_experts_sort) with its own W [experts, n_out, n_in] and B [experts, n_out] (or None)."""
    device, (rows, n_in) = _current(X), X.shape
    at, experts = _experts_of(offsets, device)
    if W.dim() != 3:
        raise ValueError("fpdt_tw: W must be [experts, n_out, n_in], got %s" % (tuple(W.shape),))
    n_out = W.size(1)
    _sizes(n_in, n_out)
    out = (rows, n_out)
    _check(load().fpdt_tw_experts_affine_fwd(_half("X", X, X.shape, device), _half("W", W, (experts, n_out, n_in), device), _half("B", B, (experts, n_out), device),
                                             _half("R", R, out, device), _half("Z", Z, out, device), _half("Y", Y, out, device), at, rows, experts, n_in, n_out, act, join,
                                             _raw_stream(stream, device)))


def fpdt_tw_experts_linear_bwd(X, W, dY, dX, dW, offsets, stream=None):
    """dX (bf16, written, or None) = dY W of each row's expert;  dW (fp32 [experts, n_out, n_in], accumulated into, or None) += dY^T X over its rows."""
    device, (rows, n_in) = _current(X), X.shape
    at, experts = _experts_of(offsets, device)
    if W.dim() != 3:
        raise ValueError("fpdt_tw: W must be [experts, n_out, n_in], got %s" % (tuple(W.shape),))
    n_out = W.size(1)
    _sizes(n_in, n_out)
    _check(load().fpdt_tw_experts_linear_bwd(_half("X", X, X.shape, device), _half("W", W, (experts, n_out, n_in), device), _half("dY", dY, (rows, n_out), device),
                                             _half("dX", dX, X.shape, device), None if dW is None else _expect("dW", dW, W.shape, torch.float32, device), at, rows,
                                             experts, n_in, n_out, _raw_stream(stream, device)))


class _Param(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64)] + [(k, ctypes.c_void_p) for k in ("g", "p", "w", "m", "v", "m_exp", "v_exp", "m_value", "v_value")] \
        + [("weight_decay", ctypes.c_double)]


class FpdtTwParams:
    """A list of tensors for fpdt_tw_grad_norm and fpdt_tw_adamw_*: lists of the same length, made once and kept as long as
    the tensors are where they are.  g: fp32 or bf16; p: fp32; w: bf16 (each or all may be None); m, v: fp32, or uint8 with m_exp, v_exp [ceil(n / 128)]
    (all zero at first); m_value, v_value: bf16, for fpdt_tw_adamw_unpack; weight_decay: a number, or one for each tensor.  The
    tensors stay alive as long as this object does, whatever becomes of the lists that they came in."""

    def __init__(self, g, p=None, m=None, v=None, w=None, m_exp=None, v_exp=None, m_value=None, v_value=None, weight_decay=0.0):
        for k, tensors in (("g", g), ("p", p), ("m", m), ("v", v), ("w", w), ("m_exp", m_exp), ("v_exp", v_exp), ("m_value", m_value), ("v_value", v_value)):
            if tensors is not None and (len(tensors) != len(g) or not len(g)):
                raise ValueError("fpdt_tw: %d tensors of g, but %d of %s" % (len(g), len(tensors), k))
        self.count, self.grad_dtype, self.device = len(g), _dtype_code(g[0]), g[0].device
        self.state_bits = 8 if m is not None and m[0].dtype == torch.uint8 else 32
        state = torch.uint8 if self.state_bits == 8 else torch.float32
        given = {"g": (g, g[0].dtype), "p": (p, torch.float32), "w": (w, torch.bfloat16), "m": (m, state), "v": (v, state), "m_exp": (m_exp, torch.uint8),
                 "v_exp": (v_exp, torch.uint8), "m_value": (m_value, torch.bfloat16), "v_value": (v_value, torch.bfloat16)}
        given = {k: x for k, x in given.items() if x[0] is not None}
        if not isinstance(weight_decay, (list, tuple)):
            weight_decay = [weight_decay] * self.count
        if len(weight_decay) != self.count:
            raise ValueError("fpdt_tw: %d tensors of g, but %d values of weight_decay" % (self.count, len(weight_decay)))
        self.array, taken = (_Param * self.count)(), []
        for i in range(self.count):
            n = g[i].numel()
            self.array[i].n, self.array[i].weight_decay = n, weight_decay[i]
            for k, (tensors, dtype) in given.items():
                t = tensors[i]
                if t is None and k == "w":
                    continue
                want = -(-n // FPDT_TW_STATE_BLOCK) if k in ("m_exp", "v_exp") else n
                if t.dtype != dtype or t.device != self.device:
                    raise TypeError("fpdt_tw: %s[%d] must be %s on %s, got %s on %s" % (k, i, dtype, self.device, t.dtype, t.device))
                if t.numel() != want or not t.is_contiguous():
                    raise ValueError("fpdt_tw: %s[%d] must be contiguous and have %d elements, got %s" % (k, i, want, tuple(t.shape)))
                setattr(self.array[i], k, t.data_ptr())
                if n:
                    taken.append((t.data_ptr(), t.data_ptr() + _nbytes(t), "%s[%d]" % (k, i)))
        taken.sort()
        for a, b in zip(taken, taken[1:]):
            if b[0] < a[1]:
                raise ValueError("fpdt_tw: %s and %s overlap" % (a[2], b[2]))
        # the tensors, not the caller's lists of them, and the memory that they have now: neither a list that is changed later nor a
        # `.data` that is replaced leaves an address of freed memory here
        self._keep = [(t, t.untyped_storage()) for tensors, _ in given.values() for t in tensors if t is not None]
        self.address = ctypes.addressof(self.array)

    def _args(self):
        if self.device.type != "cuda" or self.device.index != torch.cuda.current_device():
            raise ValueError("fpdt_tw: tensors must be on the current device, got %s" % self.device)
        return self.address, self.count


def fpdt_tw_grad_norm_workspace_bytes(params) -> int:
    return int(load().fpdt_tw_grad_norm_workspace_bytes(params.count))


def fpdt_tw_grad_norm(params, max_norm, out, workspace, stream=None):
    """out (fp32 [2]): norm of all gradients, and the factor that brings it down to max_norm."""
    args, device = params._args(), params.device.index
    _check(load().fpdt_tw_grad_norm(*args, params.grad_dtype, max_norm, _expect("out", out, (2,), torch.float32, device), *_room(workspace, device),
                                    _raw_stream(stream, device)))


def fpdt_tw_adamw_step(params, lr, beta1, beta2, eps, step, lr_dev=None, step_dev=None, grad_scale=None, seed=0, flags=0, stream=None):
    """One step.  lr_dev (fp32), step_dev (int64), grad_scale (fp32): one value each on the device, or None; lr and step are
    ignored where lr_dev and step_dev are given.  seed (8-bit states): a number of its own for each list of a model."""
    args, device, at = params._args(), params.device.index, []
    for name, t, dtype in (("lr_dev", lr_dev, torch.float32), ("step_dev", step_dev, torch.int64), ("grad_scale", grad_scale, torch.float32)):
        if t is not None and (t.dtype != dtype or t.get_device() != device or t.numel() != 1):
            raise ValueError("fpdt_tw: %s must be one %s on %s" % (name, dtype, params.device))
        at.append(None if t is None else t.data_ptr())
    _check(load().fpdt_tw_adamw_step(*args, params.grad_dtype, params.state_bits, lr, beta1, beta2, eps, step, *at, seed & 0xffffffff, flags,
                                     _raw_stream(stream, device)))


def fpdt_tw_adamw_unpack(params, stream=None):
    """m_value and v_value of the list: what its 8-bit states stand for."""
    args = params._args()
    if params.state_bits != 8:
        raise ValueError("fpdt_tw: the list's states are in 32 bits")
    _check(load().fpdt_tw_adamw_unpack(*args, _raw_stream(stream, params.device.index)))
