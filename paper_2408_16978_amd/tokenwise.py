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
