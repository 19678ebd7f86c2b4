"""The training path far from magnitudes of order one: against the fp64 oracle, within what the roundings allow."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import train_util as tu
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    import paper_2401_04044_amd as m
    return m


# ---------------------------------------------------------------- the norm's backward pass

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 520, 1536, 8200])
def test_rmsnorm_backward_wherever_the_norm_itself_is_defined(ff, d, dtype):
    """Rows whose r^3 leaves fp32 although r, and the result, do not: the forward pass has them right, so has this."""
    rng = np.random.default_rng(d)
    eps = float(np.float32(1e-32))
    scale = np.array([1e-14, 1e-13, 1.0, 1e13, 1e15, 1e16, 0.0])[:, None]
    x = (rng.standard_normal((len(scale), d)) * scale).astype(np.float32)
    dn = gu.dev(rng.standard_normal(x.shape), dtype)
    dnh = gu.host(dn)
    r = 1 / np.sqrt((x.astype(np.float64) ** 2).mean(1, keepdims=True) + eps)
    # as for rows of order one: fp32 sums of d terms, each term of the result a few roundings
    m = np.abs(r * dnh) + np.abs(x) * r ** 3 * (np.abs(x) * np.abs(dnh)).mean(1, keepdims=True)
    dx = ff.token_rmsnorm_backward(torch.from_numpy(x).cuda(), dn, eps)
    want = orc.token_rmsnorm_backward(x, dnh, eps)
    tu.assert_within(gu.host(dx), want, ((2 * tu.g(d) + 8 * 2.0 ** -24) * m, tu.U["f32"]), f"rmsnorm backward {d} {dtype}")


# ---------------------------------------------------------------- the kept derivatives of a bf16 layer

@pytest.mark.parametrize("which", ["tokens", "up", "gate"])
@pytest.mark.parametrize("log2", [-17, -20, -24, -34, 8])
def test_small_and_large_factors_keep_their_precision(ff, which, log2, monkeypatch):
    """Tokens or weights of any size: the factors dH/dU, dH/dG follow them, with a relative error of at most 2^-10."""
    T, d, f = 33, 64, 203
    host = list(tu.make_layer(np.random.default_rng(40), d, f, True, T, "bf16"))
    i = ("tokens", "up", "gate").index(which)
    host[i] = host[i] * np.float32(2.0 ** log2)
    X, W1, Wg, W2, dY = host
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    dev = tu.to_dev(host, "bf16")
    _, kept = ff.dense_forward(desc, *dev[:4], want_saved=True)
    dX, g = ff.dense_backward(desc, *dev[:4], kept, dev[4])
    _, tape = orc.dense_forward(X, W1, Wg, W2)
    want_dX, want = orc.dense_backward(X, W1, Wg, W2, tape, dY)
    monkeypatch.setitem(tu.UD, tu.U["bf16"], (2.0 ** -10, 0.0))
    b = tu.dense_bounds(X, W1, Wg, W2, tape, dY, tu.U["bf16"], tu.U["bf16"])
    for name, got, ref in [("dX", dX, want_dX)] + [(k, g[k], want[k]) for k in ("W1", "Wg", "W2")]:
        tu.assert_within(gu.host(got), ref, b[name], f"{which} 2^{log2} {name}")
        assert gu.relf(gu.host(got), ref) < gu.TOL["bf16"], (which, log2, name)


def _one_to_one(ff, act, dtype, z, u=None):
    """A layer whose neuron j sees exactly z[j] (and u[j]): returns H and what the backward pass multiplies dH = 1 with."""
    d = f = len(z)
    zero = np.zeros((d, f))
    X, dY = np.zeros((1, d)), np.ones((1, d))
    X[0, 0] = 1.0
    Wz, Wu = zero.copy(), zero.copy()
    Wz[0] = z
    if u is not None:
        Wu[0] = u
    W1, Wg = (Wz, None) if u is None else (Wu, Wz)
    desc = ff.make_desc(d, f, act, dtype)
    dev = [gu.dev(a, dtype) for a in (X, W1, Wg, np.eye(d), dY)]
    Y, kept = ff.dense_forward(desc, *dev[:4], want_saved=True, y_f32=True)
    _, g = ff.dense_backward(desc, *dev[:4], kept, dev[4], grad_f32=True)
    return gu.host(Y)[0], gu.host(g["W1"])[0], None if u is None else gu.host(g["Wg"])[0]


def test_kept_factors_from_the_smallest_to_the_largest(ff):
    """dH/dU = silu(z) for z from 2^-60 to 65504, through dU's own rounding to bf16."""
    import workloads as wl
    z = wl.bf16_round(np.exp2(np.linspace(-60, 15.9, 128)).astype(np.float32)).astype(np.float64)
    z[1::2] *= -1
    z[5], z[7] = 0.0, -65280.0
    H, dU, dG = _one_to_one(ff, "swiglu", "bf16", z, np.ones(128))
    s = 1 / (1 + np.exp(-np.clip(z, -600, 600)))
    silu, slope = z * s, s * (1 + z * (1 - s))
    # factor, dU, and the sigmoid's own error (an exponential and a reciprocal of a few units, e^-z off by |z| 2^-23)
    act = (np.minimum(np.abs(z), 200) + 8) * 2.0 ** -23
    kept = np.where(np.abs(silu) >= 2.0 ** -44, 2.0 ** -10, np.where(np.abs(silu) >= 2.0 ** -48, 2.0 ** -8, 1.0))
    assert (np.abs(dU - silu) <= (1.01 * (2.0 ** -8 + kept) + act) * np.abs(silu) + 2.0 ** -66).all()
    assert dU[5] == 0.0 and np.isfinite(dU).all()
    assert (np.abs(dG - slope) <= (1.01 * (2.0 ** -8 + 2.0 ** -10)) * np.abs(slope) + 2e-6 * (1 + np.minimum(np.abs(z), 200))).all()
    H, dU, _ = _one_to_one(ff, "swiglu", "bf16", np.array([1e-3, 65536.0, 1e9, 1.0, 2.0, 3.0, 4.0, 5.0]), np.ones(8))
    assert np.isfinite(H).all() and list(np.isfinite(dU)) == [True, False, False] + [True] * 5


# ---------------------------------------------------------------- GeLU's lower tail

def _phi(z):
    import math
    return np.array([0.5 * math.erfc(-t / math.sqrt(2.0)) for t in z]), np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def test_gelu_in_fp32_is_accurate_in_its_tail(ff):
    """z from -12 to 4.  The arguments of erfc and exp are off by 2^-23 of z / sqrt 2 and z^2 / 2, which moves either by
    z^2 2^-23 of its value at most; the functions themselves and the products add less than 32 units."""
    z = np.linspace(-12, 4, 256).astype(np.float32).astype(np.float64)
    H, slope, _ = _one_to_one(ff, "gelu", "f32", z)
    cdf, phi = _phi(z)
    tol = (2 * z * z + 32) * 2.0 ** -23
    assert (np.abs(H - z * cdf) <= tol * np.abs(z * cdf)).all()
    # (the slope is a difference of two such terms below zero)
    assert (np.abs(slope - (cdf + z * phi)) <= tol * (cdf + np.abs(z) * phi)).all()


def test_gelu_in_bf16_in_its_tail(ff):
    """Phi is off by 1e-7 at most, everywhere; H and the kept slope are rounded to bf16 and to 2^-10."""
    import workloads as wl
    z = wl.bf16_round(np.linspace(-12, 4, 256).astype(np.float32)).astype(np.float64)
    H, slope, _ = _one_to_one(ff, "gelu", "bf16", z)
    cdf, phi = _phi(z)
    assert (np.abs(H - z * cdf) <= 2.0 ** -8 * np.abs(z * cdf) + 1.01e-7 * np.abs(z)).all()
    assert (np.abs(slope - (cdf + z * phi)) <= 1.01 * (2.0 ** -8 + 2.0 ** -10) * np.abs(cdf + z * phi) + 2e-7 * (1 + np.abs(z))).all()


# ---------------------------------------------------------------- clipping

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("limit", [1.0, 1e-6, 1e-20, 1e-35, 2.0 ** -126])
def test_clipping_by_a_factor_below_the_normal_numbers(ff, limit, dtype):
    """Gradients of 1e35 and 1e20 scaled by max_norm / norm, which is subnormal or less: the results are ordinary numbers."""
    g = torch.full((4099,), 1e35, dtype=gu.TDT[dtype], device="cuda")
    g[::3] = -1e20
    g[1] = 0.0
    host = gu.host(g)
    norm, flag, (out,) = ff.clip_grad_norm([g.clone()], limit)
    limit = float(np.float32(limit))
    want = host * (limit / orc.grad_norm([host]))
    # the norm, the factor and the product are rounded to fp32 (at their subnormal end by half of 2^-149), the result to its type
    step = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    assert int(flag) == 0
    assert (np.abs(gu.host(out) - want) <= (3 * 2.0 ** -24 + tu.U[dtype]) * np.abs(want) + step).all()
    # in two halves, into other buffers: the same bits
    two = ff.grad_clip([g[:2048], g[2048:]], norm, limit, out=[torch.empty_like(g[:2048]), torch.empty_like(g[2048:])])
    assert torch.equal(torch.cat(two), out)


def test_silu_in_fp32_neuron_by_neuron(ff):
    """An exponential, a division and two products: 16 half steps of the value, of 1 + |z| for the slope (which has a zero)."""
    z = np.linspace(-80, 40, 256).astype(np.float32).astype(np.float64)
    H, dU, dG = _one_to_one(ff, "swiglu", "f32", z, np.ones(256))
    s = 1 / (1 + np.exp(-z))
    assert (np.abs(H - z * s) <= 16 * 2.0 ** -24 * np.abs(z * s)).all()
    assert (np.abs(dU - z * s) <= 16 * 2.0 ** -24 * np.abs(z * s)).all()
    slope = s * (1 + z * (1 - s))
    assert (np.abs(dG - slope) <= 16 * 2.0 ** -24 * s * (1 + np.abs(z))).all()
