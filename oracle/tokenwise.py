"""fp64 oracle of the token-wise neighbours (Sec. 5.4): plain definitions in numpy.

TEST INFRASTRUCTURE ONLY.  Chunking does not change what these operations compute, so the
oracle is the unchunked definition; inputs are the stored bits widened to fp64.
"""
import math

import numpy as np


def cross_entropy(H, W, target, grad_scale=1.0):
    """logits = H W^T; lse_r = log sum_v exp(logits_r[v]) (max-subtracted); loss_r = lse_r -
    logits_r[target_r]; gradient of sum_r grad_scale * loss_r with respect to H and W.
    Returns dict loss [rows], lse [rows], dH [rows, hidden], dW [vocab, hidden]."""
    H = np.asarray(H, dtype=np.float64)
    W = np.asarray(W, dtype=np.float64)
    t = np.asarray(target, dtype=np.int64)
    logits = H @ W.T
    m = logits.max(axis=1, keepdims=True)
    lse = (m + np.log(np.exp(logits - m).sum(axis=1, keepdims=True)))[:, 0]
    rows = np.arange(H.shape[0])
    loss = lse - logits[rows, t]
    G = np.exp(logits - lse[:, None])
    G[rows, t] -= 1.0
    G *= grad_scale
    return {"loss": loss, "lse": lse, "dH": G @ W, "dW": G.T @ H}


def linear(X, W, dY=None):
    """Y = X W^T (Sec. 4.1, the projection of one sequence chunk); with dY also dX = dY W and
    dW = dY^T X.  Returns dict Y [, dX, dW]."""
    X = np.asarray(X, dtype=np.float64)
    W = np.asarray(W, dtype=np.float64)
    out = {"Y": X @ W.T}
    if dY is not None:
        dY = np.asarray(dY, dtype=np.float64)
        out["dX"] = dY @ W
        out["dW"] = dY.T @ X
    return out


_erf = np.vectorize(math.erf, otypes=[np.float64])


def ffn(X, W1, W2, W3=None, dY=None):
    """Feed-forward block.  W3 is None: Y = gelu(X W1^T) W2^T with gelu(a) = a Phi(a), Phi the
    standard normal CDF.  Otherwise Y = (silu(X W1^T) * (X W3^T)) W2^T, silu(a) = a / (1 + e^-a).
    With dY also the gradients of sum(Y * dY): dX, dW1, dW2 (and dW3)."""
    X = np.asarray(X, dtype=np.float64)
    W1 = np.asarray(W1, dtype=np.float64)
    W2 = np.asarray(W2, dtype=np.float64)
    A = X @ W1.T
    if W3 is None:
        Phi = 0.5 * (1.0 + _erf(A / math.sqrt(2.0)))
        Hh = A * Phi
    else:
        W3 = np.asarray(W3, dtype=np.float64)
        B = X @ W3.T
        sg = 1.0 / (1.0 + np.exp(-A))
        Hh = A * sg * B
    out = {"Y": Hh @ W2.T}
    if dY is None:
        return out
    dY = np.asarray(dY, dtype=np.float64)
    dHh = dY @ W2
    out["dW2"] = dY.T @ Hh
    if W3 is None:
        phi = np.exp(-0.5 * A * A) / math.sqrt(2.0 * math.pi)
        dA = dHh * (Phi + A * phi)
        out["dX"] = dA @ W1
    else:
        dA = dHh * B * (sg + A * sg * (1.0 - sg))
        dB = dHh * A * sg
        out["dX"] = dA @ W1 + dB @ W3
        out["dW3"] = dB.T @ X
    out["dW1"] = dA.T @ X
    return out


def rope_freqs(rot, base):
    return np.asarray(base, dtype=np.float64) ** (-2.0 * np.arange(rot // 2) / rot)


def rope(X, positions, freqs, amplitude=1.0, interleaved=False, inverse=False):
    """X [rows, heads, D]: pair i of the first 2 len(freqs) channels of every head, as a complex number
    (channels 2i, 2i+1, or i, i + rot/2), times amplitude * exp(1j * position * freqs[i]) (its conjugate
    with `inverse`, the transpose)."""
    X = np.array(X, dtype=np.float64)
    half = len(freqs)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64)
    unit = amplitude * np.exp((-1j if inverse else 1j) * angle)[:, None, :]
    a, b = (np.s_[..., 0:2 * half:2], np.s_[..., 1:2 * half:2]) if interleaved else (np.s_[..., :half], np.s_[..., half:2 * half])
    z = (X[a] + 1j * X[b]) * unit
    X[a], X[b] = z.real, z.imag
    return X


def norm(S, W, B=None, eps=0.0, layer=False, dY=None, dR=None, stats=None):
    """Rows of S normalised: by their root mean square, or (layer) by mean and standard deviation.  `stats`
    [1 or 2, rows] takes the place of the statistics of S.  With dY also dX (plus dR), dW, dB."""
    S, W = np.asarray(S, dtype=np.float64), np.asarray(W, dtype=np.float64)
    mean = S.mean(axis=1) if layer else np.zeros(len(S))
    rstd = 1.0 / np.sqrt(((S - mean[:, None]) ** 2).mean(axis=1) + eps)
    if stats is not None:
        stats = np.asarray(stats, dtype=np.float64)
        mean, rstd = (stats[0], stats[1]) if layer else (mean, stats[0])
    U = (S - mean[:, None]) * rstd[:, None]
    out = {"Y": U * W + (0.0 if B is None else np.asarray(B, dtype=np.float64)), "U": U, "stats": np.stack([mean, rstd] if layer else [rstd])}
    if dY is not None:
        dY = np.asarray(dY, dtype=np.float64)
        H = dY * W
        level = H.mean(axis=1, keepdims=True) if layer else 0.0
        out["dX"] = rstd[:, None] * (H - level - U * (H * U).mean(axis=1, keepdims=True)) + (0.0 if dR is None else np.asarray(dR, dtype=np.float64))
        out["dW"], out["dB"] = (dY * U).sum(axis=0), dY.sum(axis=0)
    return out


def grad_norm(grads, max_norm):
    n = math.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    return n, (min(1.0, max_norm / (n + 1e-6)) if math.isfinite(n) else math.nan)


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, scale=1.0):
    p, g, m, v = (np.asarray(a, dtype=np.float64) for a in (p, g, m, v))
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    move = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * (move + weight_decay * p), m, v


def _mix(x):
    x ^= x >> 15
    x = x * 0xB7E15163 % 2 ** 32
    x ^= x >> 13
    x = x * 0x93C467E3 % 2 ** 32
    return x ^ (x >> 16)


def state_chances(n, seed, step, k):
    """Two numbers in [0, 1) for each element of tensor k, in 1 / 65536: for m and for v."""
    key = _mix(_mix(_mix(seed ^ 0x243F6A88) ^ (step * 0x9E3779B1 % 2 ** 32)) ^ (k * 0x85A308D3 % 2 ** 32))
    r = np.array([_mix((i * 0x9E3779B1 % 2 ** 32) ^ key) for i in range(n)], dtype=np.int64)
    return (r % 65536) / 65536.0, (r // 65536) / 65536.0


def state_value(code, exp, signed):
    """What 8-bit codes stand for, blocks of 128 with an exponent byte each."""
    code, e = np.asarray(code, dtype=np.int64), np.repeat(np.asarray(exp, dtype=np.int64), 128)[:len(code)]
    mag, span = (code % 128, 15) if signed else (code, 31)
    x = np.where(mag > 0, (1 + (mag % 8) / 8.0) * 2.0 ** (e - 127.0 - span + mag // 8), 0.0)
    return np.where(e == 255, np.nan, np.where(signed & (code > 127), -x, x))


def state_rounded(x, chance, signed):
    """x rounded up in size where `chance` is at least what is missing to the next code, else down; also how far (in
    steps) the decision is from the other one, and the exponent bytes."""
    x = np.asarray(x, dtype=np.float64)
    size, span, n = np.abs(x), 15 if signed else 31, len(x)
    blocks = -(-n // 128)
    top = np.zeros(blocks * 128)
    top[:n] = size
    top = top.reshape(blocks, 128).max(axis=1)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(top))
        e = np.where(top > 1.875 * 2.0 ** e, e + 1, e)
        exp = np.where(np.isfinite(top), np.maximum(e + 127, 40), 255)
        exp = np.minimum(exp, 255)
        least = np.repeat(1.125 * 2.0 ** (exp - 127 - span), 128)[:n]
        grid = 2.0 ** (np.floor(np.log2(np.maximum(size, 1e-300))) - 3)
    with np.errstate(invalid="ignore"):
        up = size / grid + chance
    low = chance * least < size if signed else size > 0
    value = np.where(size >= least, np.floor(up) * grid, np.where(low, least, 0.0))
    slack = np.where(size >= least, np.abs(up - np.round(up)), np.abs(chance - size / least) if signed else 1.0)
    return np.where(np.repeat(exp, 128)[:n] == 255, np.nan, value * np.sign(x)), slack, exp.astype(np.int64)
