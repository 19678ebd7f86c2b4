"""The device's 64-bit reference against the numpy oracle, and its bounds against a layer rounded as the library rounds it (no GPU)."""
import numpy as np
import pytest
import torch

import train_ref as tr
from oracle import train_oracle as orc


@pytest.mark.parametrize("gated", [False, True])
def test_reference_is_the_oracle(gated):
    gen = torch.Generator()
    gen.manual_seed(3)
    ts = [None if t is None else t.double() for t in tr.make_layer(gen, 24, 37, gated, 11, "f32")]
    out, _ = tr.reference(*ts)
    X, W1, Wg, W2, dY = (None if t is None else t.numpy() for t in ts)
    Y, kept = orc.dense_forward(X, W1, Wg, W2)
    dX, grads = orc.dense_backward(X, W1, Wg, W2, kept, dY)
    for k, want in [("Y", Y), ("dX", dX)] + [(k, w) for k, w in grads.items() if w is not None]:
        assert np.allclose(out[k].numpy(), want, rtol=1e-12, atol=1e-14), k


@pytest.mark.parametrize("gated", [False, True])
def test_bounds_hold_the_roundings_and_no_more(gated):
    """H, dU, dG in bf16 and the factors off by 2^-10: within; three of their steps off in one neuron: not."""
    gen = torch.Generator()
    gen.manual_seed(4)
    X, W1, Wg, W2, dY = (None if t is None else t.double() for t in tr.make_layer(gen, 64, 96, gated, 9, "bf16"))
    want, inner = tr.reference(X, W1, Wg, W2, dY)
    b = tr.bounds(X, W1, Wg, W2, dY, inner, "bf16")
    z, up, H, dz, du, dH = inner
    r = lambda t: t.bfloat16().double()
    for wrong in (False, True):
        k = 1 + 2.0 ** -10
        H8, D = r(H), [r(dH * t * k) for t in ((dz,) if Wg is None else (du, dz))]
        if wrong:
            H8[:, 5] *= 1 + 2.0 ** -5
            D[0][:, 5] *= 1 + 2.0 ** -5
        got = {"Y": H8 @ W2, "W2": H8.t() @ dY, "W1": X.t() @ D[0],
               "dX": D[0] @ W1.t() + (0 if Wg is None else D[1] @ Wg.t())}
        if Wg is not None:
            got["Wg"] = X.t() @ D[1]
        for name in got:
            if not wrong:
                tr.assert_within(got[name], want[name], b[name], 0.0, name)
        if wrong:
            for name in ("W1", "W2"):
                with pytest.raises(AssertionError):
                    tr.assert_within(got[name], want[name], b[name], 0.0, name)
