"""The training path in 64 bits on any device, with bounds on what the library's roundings may change, entry by entry: what
train_util.py has in numpy, for sizes that need the GPU's speed.  The bounds' derivation is the same, but that the kept
derivatives of a bf16 layer are off by at most 2^-10 of their value.  (Activations are allowed 1e-6, eight units of fp32:
what their forms do beyond that, test_gpu_train_range.py holds neuron by neuron.)"""
import math

import torch

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
KEPT = {"bf16": 2.0 ** -10, "f32": 2.0 ** -24}
A = 1e-6


def g(n):
    return n * 2.0 ** -23


def reference(X, W1, Wg, W2, dY):
    """Outputs and their bounds' ingredients: all arguments float64 on one device, Wg None un-gated."""
    if Wg is None:
        z, up = X @ W1, None
        cdf = 0.5 * torch.special.erfc(z * -math.sqrt(0.5))
        phi = torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        H, dz, du = z * cdf, cdf + z * phi, None
    else:
        z, up = X @ Wg, X @ W1
        s = torch.sigmoid(z)
        H, dz, du = z * s * up, up * s * (1 + z * (1 - s)), z * s
    dH = dY @ W2.t()
    out = {"Y": H @ W2, "W2": H.t() @ dY}
    if Wg is None:
        dU = dH * dz
        out["dX"], out["W1"] = dU @ W1.t(), X.t() @ dU
    else:
        dU, dG = dH * du, dH * dz
        out["dX"], out["W1"], out["Wg"] = dU @ W1.t() + dG @ Wg.t(), X.t() @ dU, X.t() @ dG
    return out, (z, up, H, dz, du, dH)


def bounds(X, W1, Wg, W2, dY, inner, dtype):
    """|error| of Y, dX and the weights' gradients before their own rounding."""
    u, ud = U[dtype], KEPT[dtype]
    z, up, H, dz, du, dH = (None if t is None else t.abs() for t in inner)
    X, W1, W2, dY = X.abs(), W1.abs(), W2.abs(), dY.abs()
    T, d = X.shape
    f = H.shape[1]
    a_h, a_s = A, A * (1 + z)     # the activations' own errors: of h / z and of the slope
    if Wg is None:
        e = g(d) * (X @ W1)
        eH = 1.13 * e + a_h * z + u * H
        parts = [(dz, 0.8 * e + a_s + ud * dz, W1, "W1")]
    else:
        Wg = Wg.abs()
        ez, eu = g(d) * (X @ Wg), g(d) * (X @ W1)
        silu = 1.1 * ez + a_h * z
        eH = silu * (up + eu) + du * eu + u * H
        parts = [(du, silu + ud * du, W1, "W1"), (dz, (0.5 * ez + a_s) * (up + eu) + 1.1 * eu + ud * dz, Wg, "Wg")]
    M = dY @ W2.t()
    out = {"Y": eH @ W2 + g(f) * ((H + eH) @ W2), "W2": eH.t() @ dY + g(T) * ((H + eH).t() @ dY), "dX": 0.0}
    for v, ev, W, name in parts:
        m = dH * v
        em = g(d) * M * (v + ev) + dH * ev + u * m
        out["dX"] = out["dX"] + em @ W.t() + g(f * len(parts)) * ((m + em) @ W.t())
        out[name] = X.t() @ em + g(T) * (X.t() @ (m + em))
    return {k: 1.05 * b for k, b in out.items()}


def assert_within(got, want, bound, u, what):
    """Entry by entry: the bound, and half a step of the output's type."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), (what, "non-finite")
    allowed = bound + u * (want.abs() + bound) + 1e-37
    off = (got - want).abs()
    if not bool((off <= allowed).all()):
        i = int((off / allowed).argmax())
        raise AssertionError((what, i, float(got.flatten()[i]), float(want.flatten()[i]), float(allowed.flatten()[i])))


def make_layer(gen, d, f, gated, T, dtype):
    """Tokens N(0, 1), weights that keep pre-activations of order 1, 5 % of the neurons scaled by 8, in the storage type."""
    dev, dt = gen.device, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]

    def normal(shape, scale):
        return torch.randn(shape, generator=gen, device=dev) * scale

    heavy = 1 + 7 * (torch.rand(f, generator=gen, device=dev) < 0.05).float()
    W1, W2 = normal((d, f), d ** -0.5) * heavy, normal((f, d), d ** -0.5)
    Wg = (normal((d, f), d ** -0.5) * heavy).to(dt) if gated else None
    return normal((T, d), 1.0).to(dt), W1.to(dt), Wg, W2.to(dt), normal((T, d), 1e-2).to(dt)
