"""Plain fp64 numpy forms of the training path: the uncompressed feed-forward layer with its backward pass,
the backward pass of the per-token RMS norm, the norm over all gradients and clipping, and a stack of
pre-norm layers.  Weights as the library takes them: W1, Wg [d, f], W2 [f, d]; Wg None un-gated."""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def _f8(a):
    return None if a is None else np.asarray(a, np.float64)


def activation(z, u=None):
    """(H, dH/dz, dH/du): gelu(z), or silu(z) u."""
    z = _f8(z)
    if u is None:
        cdf = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
        return z * cdf, cdf + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi), None
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-z))
    return z * s * u, u * s * (1.0 + z * (1.0 - s)), z * s


def dense_forward(X, W1, Wg, W2):
    """(Y, kept): kept = (z, u, H, dH/dz, dH/du)."""
    X, W1, Wg, W2 = _f8(X), _f8(W1), _f8(Wg), _f8(W2)
    z, u = (X @ W1, None) if Wg is None else (X @ Wg, X @ W1)
    H, dz, du = activation(z, u)
    return H @ W2, (z, u, H, dz, du)


def dense_backward(X, W1, Wg, W2, kept, dY):
    """(dX, {"W1", "Wg", "W2"})."""
    X, W1, Wg, W2, dY = _f8(X), _f8(W1), _f8(Wg), _f8(W2), _f8(dY)
    _, _, H, dz, du = kept
    dH = dY @ W2.T
    if Wg is None:
        dU = dH * dz
        return dU @ W1.T, {"W1": X.T @ dU, "Wg": None, "W2": H.T @ dY}
    dG, dU = dH * dz, dH * du
    return dU @ W1.T + dG @ Wg.T, {"W1": X.T @ dU, "Wg": X.T @ dG, "W2": H.T @ dY}


def token_rmsnorm(x, eps):
    x = _f8(x)
    return x / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)


def token_rmsnorm_backward(x, dn, eps, residual=None):
    x, dn = _f8(x), _f8(dn)
    r = 1.0 / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)
    dx = r * dn - x * r ** 3 * (x * dn).mean(axis=1, keepdims=True)
    return dx if residual is None else _f8(residual) + dx


def grad_norm(grads):
    return math.sqrt(math.fsum(float((_f8(g) ** 2).sum()) for g in grads))


def grad_clip(grads, norm, max_norm):
    k = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return [_f8(g) * k for g in grads]


def stack_forward(layers, x, eps):
    """layers: (W1, Wg, W2) each.  Returns (x behind the last layer, tape)."""
    x, tape = _f8(x), []
    for W in layers:
        n = token_rmsnorm(x, eps)
        Y, kept = dense_forward(n, *W)
        tape.append((x, n, kept))
        x = x + Y
    return x, tape


def stack_backward(layers, tape, dx, eps):
    """(gradient of the stream in front of the first layer, gradients per layer)."""
    dx, grads = _f8(dx), [None] * len(layers)
    for l in range(len(layers) - 1, -1, -1):
        x, n, kept = tape[l]
        dn, grads[l] = dense_backward(n, *layers[l], kept, dx)
        dx = token_rmsnorm_backward(x, dn, eps, dx)
    return dx, grads

