"""The training path's oracle against differences and by hand; the host's checks of arguments (no GPU)."""
import ctypes
import math

import numpy as np
import pytest

from oracle import train_oracle as orc


def _layers(rng, n, d, f, gated):
    return [(rng.standard_normal((d, f)) / math.sqrt(d), rng.standard_normal((d, f)) / math.sqrt(d) if gated else None,
             rng.standard_normal((f, d)) / math.sqrt(d)) for _ in range(n)]


def _check_differences(fun, arrays, grads, rng, h=1e-5):
    """Directional derivatives of the scalar fun() along random directions, central differences (error h^2)."""
    for a, ga in zip(arrays, grads):
        for _ in range(3):
            v = rng.standard_normal(a.shape)
            a += h * v
            hi = fun()
            a -= 2 * h * v
            lo = fun()
            a += h * v
            want = (hi - lo) / (2 * h)
            assert abs(float((ga * v).sum()) - want) < 1e-7 * max(1.0, abs(want)) * math.sqrt(a.size)


@pytest.mark.parametrize("gated", [False, True])
def test_layer_gradients_are_those_of_differences(gated):
    rng = np.random.default_rng(3)
    (W1, Wg, W2), = _layers(rng, 1, 6, 9, gated)
    X, dY = rng.standard_normal((5, 6)), rng.standard_normal((5, 6))
    Y, kept = orc.dense_forward(X, W1, Wg, W2)
    dX, g = orc.dense_backward(X, W1, Wg, W2, kept, dY)
    names = ["W1", "W2"] + (["Wg"] if gated else [])
    arr = {"W1": W1, "W2": W2, "Wg": Wg}
    _check_differences(lambda: float((orc.dense_forward(X, W1, Wg, W2)[0] * dY).sum()), [X] + [arr[k] for k in names],
                       [dX] + [g[k] for k in names], rng)


def test_activation_slopes_by_hand():
    assert orc.activation(0.0)[1] == 0.5
    h, dz, du = orc.activation(0.0, 2.0)
    assert (h, dz, du) == (0.0, 1.0, 0.0)              # silu(0) = 0, silu'(0) = 1/2
    z = 1.25
    s = 1 / (1 + math.exp(-z))
    h, dz, du = orc.activation(z, 3.0)
    assert abs(dz - 3.0 * (s + z * s * (1 - s))) < 1e-15 and abs(du - z * s) < 1e-15


def test_norm_gradient_is_that_of_differences_and_projects():
    rng = np.random.default_rng(4)
    x, dn = rng.standard_normal((4, 16)) * 3, rng.standard_normal((4, 16))
    dx = orc.token_rmsnorm_backward(x, dn, 1e-3)
    _check_differences(lambda: float((orc.token_rmsnorm(x, 1e-3) * dn).sum()), [x], [dx], rng)
    # without eps a change of length changes nothing: the gradient is orthogonal to the token
    assert np.abs((orc.token_rmsnorm_backward(x, dn, 0.0) * x).sum(1)).max() < 1e-13


@pytest.mark.parametrize("gated", [False, True])
def test_stack_gradients_are_those_of_differences(gated):
    rng = np.random.default_rng(5)
    layers = _layers(rng, 3, 6, 8, gated)
    x, dy = rng.standard_normal((4, 6)), rng.standard_normal((4, 6))
    _, tape = orc.stack_forward(layers, x, 1e-3)
    dx, grads = orc.stack_backward(layers, tape, dy, 1e-3)
    _check_differences(lambda: float((orc.stack_forward(layers, x, 1e-3)[0] * dy).sum()),
                       [x] + [W[0] for W in layers] + [W[2] for W in layers],
                       [dx] + [g["W1"] for g in grads] + [g["W2"] for g in grads], rng)


def test_clip_by_hand():
    g = [np.array([3.0]), np.array([[0.0, 4.0]]), np.zeros(0)]
    assert orc.grad_norm(g) == 5.0
    assert [c.tolist() for c in orc.grad_clip(g, 5.0, 2.5)] == [[1.5], [[0.0, 2.0]], []]
    assert orc.grad_clip(g, 5.0, 5.0)[0][0] == 3.0 and orc.grad_clip(g, math.inf, 1.0)[0][0] == 3.0


# ---------------------------------------------------------------- the library's checks, on the host

FAKE = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x1004)
HALF = ctypes.c_void_p(0x1080)      # 128-byte aligned
BIG = 1 << 40


def _forward(L, d, T=4, X=FAKE, W1=FAKE, Wg=FAKE, W2=FAKE, Y=FAKE, res=None, kept=None, ws=FAKE, n=BIG):
    return L.ffsplit_dense_forward(d, X, T, W1, Wg, W2, Y, res, 0, kept, ws, n, None)


def _backward(L, d, T=4, X=FAKE, W1=FAKE, Wg=FAKE, W2=FAKE, kept=FAKE, dY=FAKE, dX=FAKE, dW1=FAKE, dWg=FAKE, dW2=FAKE,
              flags=0, ws=FAKE, n=BIG):
    return L.ffsplit_dense_backward(d, X, T, W1, Wg, W2, kept, dY, dX, dW1, dWg, dW2, flags, ws, n, None)


def test_layer_calls_refuse_bad_arguments():
    import paper_2401_04044_amd as ff
    L, ref = ff.lib, ctypes.byref
    glu, gelu = ff.make_desc(64, 100, "swiglu", "bf16"), ff.make_desc(64, 100, "gelu", "f32")
    for call in (_forward, _backward):
        assert call(L, None) == -1
        for k in ("X", "W1", "Wg", "W2", "ws"):
            assert call(L, ref(glu), **{k: None}) == (-5 if k == "ws" else -1), k
        for k in ("X", "W1", "Wg", "W2"):
            assert call(L, ref(glu), **{k: ODD}) == -4, k
        assert call(L, ref(glu), kept=HALF) == -4 and call(L, ref(glu), ws=HALF) == -4
        assert call(L, ref(glu), T=-1) == -3 and call(L, ref(glu), T=1 << 31) == -3
        assert call(L, ref(ff.make_desc(60, 100, "swiglu", "bf16"))) == -3
        assert call(L, ref(ff.make_desc(1 << 21, 100, "swiglu", "bf16"))) == -3
        assert call(L, ref(ff.make_desc(64, 1 << 20, "swiglu", "bf16"))) == -3
        assert call(L, ref(ff.make_desc(64, 0, "swiglu", "bf16"))) == -2
        assert call(L, ref(ff.make_desc(64, 100, 3, "bf16"))) == -2
        assert call(L, ref(ff.make_desc(64, 100, "gelu", 2))) == -2
        which = ff.WS_DENSE_FORWARD if call is _forward else ff.WS_DENSE_BACKWARD
        assert call(L, ref(glu), n=ff.workspace_bytes(glu, which, 4) - 1) == -5
    assert _forward(L, ref(glu), Y=None) == -1 and _forward(L, ref(glu), Y=ODD) == -4
    assert _forward(L, ref(glu), res=ODD) == -4
    assert _backward(L, ref(glu), kept=None) == -1 and _backward(L, ref(glu), dY=None) == -1
    for k in ("dY", "dX", "dW1", "dWg", "dW2"):
        assert _backward(L, ref(glu), **{k: ODD}) == -4, k
    assert _backward(L, ref(glu), flags=4) == -2
    assert _backward(L, ref(gelu)) == -2                        # no gate, no gradient of it
    assert _forward(L, ref(glu), T=0, X=None, Y=None, ws=None) == 0


def test_gradient_calls_refuse_bad_arguments():
    import paper_2401_04044_amd as ff
    L = ff.lib
    one = lambda t, v: (t * 1)(v)
    p, c, f = one(ctypes.c_void_p, 0x1000), one(ctypes.c_int64, 8), one(ctypes.c_int32, 0)
    assert L.ffsplit_grad_norm(-1, p, c, f, FAKE, None, FAKE, BIG, None) == -3
    assert L.ffsplit_grad_norm(1, None, c, f, FAKE, None, FAKE, BIG, None) == -1
    assert L.ffsplit_grad_norm(1, one(ctypes.c_void_p, None), c, f, FAKE, None, FAKE, BIG, None) == -1
    assert L.ffsplit_grad_norm(1, one(ctypes.c_void_p, 0x1004), c, f, FAKE, None, FAKE, BIG, None) == -4
    assert L.ffsplit_grad_norm(1, p, one(ctypes.c_int64, -1), f, FAKE, None, FAKE, BIG, None) == -3
    assert L.ffsplit_grad_norm(1, p, c, one(ctypes.c_int32, 2), FAKE, None, FAKE, BIG, None) == -2
    assert L.ffsplit_grad_norm(1, p, c, f, None, None, FAKE, BIG, None) == -1
    assert L.ffsplit_grad_norm(1, p, c, f, ctypes.c_void_p(0x1002), None, FAKE, BIG, None) == -4
    assert L.ffsplit_grad_norm(1, p, c, f, FAKE, None, FAKE, 8, None) == -5
    for bad in (0.0, -1.0, math.nan):
        assert L.ffsplit_grad_clip(1, p, c, f, FAKE, bad, p, None) == -3
    assert L.ffsplit_grad_clip(1, p, c, f, None, 1.0, p, None) == -1
    assert L.ffsplit_grad_clip(1, p, c, f, FAKE, 1.0, None, None) == -1
    assert L.ffsplit_grad_clip(1, p, c, f, FAKE, 1.0, one(ctypes.c_void_p, 0x1004), None) == -4
    assert L.ffsplit_grad_clip(0, None, None, None, None, 1.0, None, None) == 0
    r = L.ffsplit_token_rmsnorm_backward
    assert r(None, FAKE, 4, 64, 1e-6, 1, None, FAKE, None, None) == -1
    assert r(FAKE, FAKE, 4, 64, 1e-6, 1, None, None, None, None) == -1
    assert r(FAKE, FAKE, 4, 60, 1e-6, 1, None, FAKE, None, None) == -3
    assert r(FAKE, FAKE, -4, 64, 1e-6, 1, None, FAKE, None, None) == -3
    assert r(FAKE, FAKE, 4, 64, 1e-6, 2, None, FAKE, None, None) == -2
    for k in (0, 1, 6, 7, 8):
        a = [FAKE, FAKE, 4, 64, 1e-6, 1, FAKE, FAKE, FAKE, None]
        a[k] = ODD
        if k in (0, 1, 6, 7, 8):
            assert r(*a) == -4
    assert r(None, None, 0, 64, 1e-6, 1, None, None, None, None) == 0


def test_stack_calls_refuse_bad_arguments():
    import paper_2401_04044_amd as ff
    L, ref = ff.lib, ctypes.byref
    d = ff.make_desc(64, 100, "swiglu", "bf16")
    good, hole, odd = ((ctypes.c_void_p * 2)(*v) for v in ((0x1000, 0x1000), (0x1000, None), (0x1000, 0x1004)))

    def fwd(W1=good, Wg=good, W2=good, x=FAKE, T=4, kept=FAKE, ws=FAKE, n=BIG, layers=2, desc=d):
        return L.ffsplit_dense_stack_forward(ref(desc), layers, W1, Wg, W2, x, T, 1e-6, kept, ws, n, None)

    def bwd(W1=good, Wg=good, W2=good, x=FAKE, T=4, kept=FAKE, ws=FAKE, n=BIG, layers=2, desc=d, dW1=good, dWg=good, dW2=good,
            flags=0, norm=None, bad=None):
        return L.ffsplit_dense_stack_backward(ref(desc), layers, W1, Wg, W2, kept, x, T, 1e-6, dW1, dWg, dW2, flags, 0.0,
                                              norm, bad, ws, n, None)

    for call in (fwd, bwd):
        for k in ("W1", "Wg", "W2"):
            assert call(**{k: None}) == -1 and call(**{k: hole}) == -1 and call(**{k: odd}) == -4, k
        assert call(x=None) == -1 and call(x=ODD) == -4 and call(kept=HALF) == -4
        assert call(ws=None) == -5 and call(ws=HALF) == -4
        assert call(n=ff.workspace_bytes(d, ff.WS_DENSE_STACK, 4) - 1) == -5
        assert call(layers=-1) == -3 and call(T=-1) == -3 and call(desc=ff.make_desc(60, 100, "swiglu", "bf16")) == -3
    assert bwd(kept=None) == -1 and bwd(flags=8) == -2
    for k in ("dW1", "dWg", "dW2"):
        assert bwd(**{k: None}) == -1 and bwd(**{k: hole}) == -1 and bwd(**{k: odd}) == -4, k
    assert bwd(norm=ctypes.c_void_p(0x1002)) == -4 and bwd(bad=ctypes.c_void_p(0x1001)) == -4
    assert fwd(layers=0, W1=None, Wg=None, W2=None, x=None, ws=None) == 0


def test_sizes_never_shrink_with_more_tokens():
    import paper_2401_04044_amd as ff
    for d in (ff.make_desc(64, 100, "swiglu", "bf16"), ff.make_desc(4096, 11008, "swiglu", "bf16"), ff.make_desc(512, 1365, "gelu", "f32")):
        for size in (lambda T: ff.workspace_bytes(d, ff.WS_DENSE_FORWARD, T), lambda T: ff.workspace_bytes(d, ff.WS_DENSE_BACKWARD, T),
                     lambda T: ff.workspace_bytes(d, ff.WS_DENSE_STACK, T), lambda T: ff.dense_kept_bytes(d, T)):
            sizes = [size(T) for T in (0, 1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 200, 500, 1000, 1024, 2000, 4096, 10000)]
            assert sizes == sorted(sizes) and sizes[1] > 0
    assert ff.dense_kept_bytes(ff.make_desc(60, 100, "gelu", "f32"), 4) == 0


def test_binding_refuses_views_types_and_shapes():
    import torch
    import paper_2401_04044_amd as ff
    d = ff.make_desc(64, 100, "swiglu", "f32")
    X, W, V = torch.zeros(4, 64), torch.zeros(64, 100), torch.zeros(100, 64)
    with pytest.raises(ValueError, match="contiguous"):
        ff.dense_forward(d, torch.zeros(64, 4).t(), W, W, V)
    with pytest.raises(TypeError):
        ff.dense_forward(d, X.double(), W, W, V)
    with pytest.raises(ValueError, match="shape"):
        ff.dense_forward(d, X, W, W, W)
    with pytest.raises(ValueError, match="bytes"):
        ff.dense_backward(d, X, W, W, V, torch.zeros(16, dtype=torch.uint8), X)
    with pytest.raises(ValueError, match="add to"):
        ff.dense_backward(d, X, W, W, V, torch.zeros(1 << 20, dtype=torch.uint8), X, accumulate=True)
    with pytest.raises(ValueError, match="no gradient"):
        ff.dense_backward(ff.make_desc(64, 100, "gelu", "f32"), X, W, None, V, torch.zeros(1 << 20, dtype=torch.uint8), X,
                          grads={"Wg": W})
    with pytest.raises(ValueError, match="contiguous"):
        ff.grad_clip([torch.zeros(8, 8)[:, ::2]], torch.zeros(1), 1.0)
    with pytest.raises(ValueError, match="tensors"):
        ff.grad_clip([X, X], torch.zeros(1), 1.0, out=[X])
    with pytest.raises(TypeError):
        ff.token_rmsnorm_backward(X, X.half())


def test_the_largest_sizes_are_refused_and_not_wrapped():
    """Rows beyond 2^28 and widths beyond 2^20: counts of them, rounded up, would pass 31 bits."""
    import paper_2401_04044_amd as ff
    L, ref = ff.lib, ctypes.byref
    for desc in (ff.make_desc(8, 8, "gelu", "bf16"), ff.make_desc(8, 8, "swiglu", "f32")):
        for T in ((1 << 28) + 1, (1 << 31) - 16, (1 << 31) - 1):
            assert _forward(L, ref(desc), T=T) == -3 and _backward(L, ref(desc), T=T) == -3
            assert ff.dense_kept_bytes(desc, T) == 0 and ff.workspace_bytes(desc, ff.WS_DENSE_FORWARD, T) == 0
        assert ff.dense_kept_bytes(desc, 1 << 28) >= (2 if desc.act == ff.ACT_GELU else 3) * 8 * (1 << 28) * (2 if desc.dtype == ff.BF16 else 4)
    for d in ((1 << 20) + 8, (1 << 31) - 8):
        assert L.ffsplit_token_rmsnorm_backward(FAKE, FAKE, 1, d, 1e-6, 1, None, FAKE, None, None) == -3


def test_binding_refuses_buffers_used_twice():
    import torch
    import paper_2401_04044_amd as ff
    d = ff.make_desc(64, 100, "gelu", "f32")
    X, dY, W, V, one = torch.zeros(4, 64), torch.zeros(4, 64), torch.zeros(64, 100), torch.zeros(100, 64), torch.zeros(1)
    saved = torch.zeros(1 << 20, dtype=torch.uint8)
    for dX in (X, dY):
        with pytest.raises(ValueError, match="dX"):
            ff.dense_backward(d, X, W, None, V, saved, dY, dX=dX)
    with pytest.raises(ValueError, match="twice"):
        ff.grad_clip([X, W, X], one, 1.0)
    with pytest.raises(ValueError, match="twice"):
        ff.grad_clip([X, dY], one, 1.0, out=[X, X])
    with pytest.raises(ValueError, match="twice"):
        ff.clip_grad_norm([X, X], 1.0)
    layers = [{"W1": W, "W2": V}, {"W1": W, "W2": V}]
    grads = [{"W1": W, "W2": V}, {"W1": W, "W2": torch.zeros(100, 64)}]
    with pytest.raises(ValueError, match="twice"):
        ff.dense_stack_backward(d, layers, saved, X, grads=grads)
