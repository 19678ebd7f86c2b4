"""How far the training path may be from exact arithmetic, entry by entry, and helpers for its tests.

The library rounds H, dU, dG and its outputs to the storage type, each by at most u times the value (u: bf16 2^-8,
fp32 2^-24), and the kept derivatives D (dH/dz, dH/du) to fp16 in bf16 layers (at most 2^-11 of the value, and 2^-25
where it is below fp16's normal range), to fp32 in fp32 layers; it forms every sum of n products in fp32: off by at
most g(n) = n 2^-23 times the sum of magnitudes, whatever the order.  Pre-activations are therefore off by
e = g(d) |X| |W|.  With |silu'| <= 1.1, |silu''| <= 0.5, |gelu'| <= 1.13, |gelu''| <= 0.8 and activations
whose sigmoid or normal distribution is off by at most a = 1e-6:
    silu: 1.1 e + a |z|      silu': 0.5 e + a (1 + |z|)      gelu, gelu' alike with their own constants
Products of two inexact factors take the other one with its error; what is left out (products of three
errors) is far below the 5 % that the bounds are widened by."""
import numpy as np

import gpu_util as gu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
UD = {2.0 ** -8: (2.0 ** -11, 2.0 ** -25), 2.0 ** -24: (2.0 ** -24, 0.0)}     # of the kept derivatives, by u
A = 1e-6


def g(n):
    return n * 2.0 ** -23


def _f8(t):
    return np.abs(np.asarray(t, np.float64))


def dense_bounds(X, W1, Wg, W2, kept, dY, u, u_grad):
    """Bounds of |error| of Y, dX (rounded with u) and the weights' gradients (rounded with u_grad)."""
    z, up, H, dz, du = kept
    dH = np.asarray(dY, np.float64) @ np.asarray(W2, np.float64).T
    X, W1, W2, dY = _f8(X), _f8(W1), _f8(W2), _f8(dY)
    z, H, dz, dH = abs(z), abs(H), abs(dz), abs(dH)
    T, d = X.shape
    f = H.shape[1]
    ud, ad = UD[u]
    if Wg is None:
        e = g(d) * (X @ W1)
        eH = 1.13 * e + A * z + u * H
        D = [(dz, 0.8 * e + A * (1 + z) + ud * dz + ad, W1, "W1")]
    else:
        Wg, up, du = _f8(Wg), abs(up), abs(du)
        ez, eu = g(d) * (X @ Wg), g(d) * (X @ W1)
        silu = 1.1 * ez + A * z
        eH = silu * (up + eu) + du * eu + u * H
        D = [(du, silu + ud * du + ad, W1, "W1"), (dz, (0.5 * ez + A * (1 + z)) * (up + eu) + 1.1 * eu + ud * dz + ad, Wg, "Wg")]
    M = dY @ W2.T                                   # dH is off by g(d) M
    out = {"Y": eH @ W2 + g(f) * ((H + eH) @ W2)}
    out["W2"] = eH.T @ dY + g(T) * ((H + eH).T @ dY)
    out["dX"] = 0.0
    for v, ev, W, name in D:
        m = dH * v
        em = g(d) * M * (v + ev) + dH * ev + u * m
        out["dX"] = out["dX"] + em @ W.T + g(f * len(D)) * ((m + em) @ W.T)
        out[name] = X.T @ em + g(T) * (X.T @ (m + em))
    return {k: (1.05 * b, u if k in ("Y", "dX") else u_grad) for k, b in out.items()}


def assert_within(got, want, bound, what):
    """Entry by entry: the bound, and half a step of the output's type."""
    b, u = bound
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), (what, "non-finite")
    off = np.abs(got - want)
    allowed = b + u * (np.abs(want) + b) + 1e-37
    worst = np.unravel_index(np.argmax(off / allowed), off.shape) if off.size else None
    assert (off <= allowed).all(), (what, worst, got[worst], want[worst], allowed[worst])


def make_layer(rng, d, f, gated, T, dtype, dy_scale=1e-2):
    """Tokens N(0, 1), weights that keep pre-activations of order 1, 5 % of the neurons scaled by 8, all exactly
    representable in the storage type."""
    import workloads as wl
    r = wl.bf16_round if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    heavy = rng.random(f) < 0.05
    s = 1.0 / np.sqrt(d)
    W1, W2 = rng.standard_normal((d, f)) * s, rng.standard_normal((f, d)) * s
    Wg = rng.standard_normal((d, f)) * s if gated else None
    for W in (W1, Wg):
        if W is not None:
            W[:, heavy] *= 8
    X, dY = rng.standard_normal((T, d)), rng.standard_normal((T, d)) * dy_scale
    return tuple(None if a is None else r(a.astype(np.float32)).astype(np.float32) for a in (X, W1, Wg, W2, dY))


def to_dev(ts, dtype):
    return [gu.dev(t, dtype) for t in ts]
