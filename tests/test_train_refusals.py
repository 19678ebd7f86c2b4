"""What the training calls refuse beyond single bad arguments (host only, no GPU)."""
import ctypes
import math

import pytest
import torch

import paper_2401_04044_amd as ff


def _layer(T=100, d=64, f=100, act="swiglu"):
    """T = d_ff, so that a token matrix has the shape of W2's gradient."""
    desc = ff.make_desc(d, f, act, "f32")
    return desc, dict(X=torch.zeros(T, d), W1=torch.zeros(d, f), Wg=torch.zeros(d, f), W2=torch.zeros(f, d),
                      saved=torch.zeros(ff.dense_kept_bytes(desc, T), dtype=torch.uint8), dY=torch.zeros(T, d))


def test_a_gradients_buffer_is_nothing_else_of_the_call():
    desc, t = _layer()
    one, two = torch.zeros(64, 100), torch.zeros(100, 64)
    flat = torch.zeros(2 * 6400)
    for W1, Wg in ((one, one), (flat[:6400].view(64, 100), flat[6396:-4].view(64, 100)), (flat[4:6404].view(64, 100), flat[:6400].view(64, 100))):
        with pytest.raises(ValueError, match="overlaps"):
            ff.dense_backward(desc, **t, grads={"W1": W1, "Wg": Wg, "W2": two})
    for k, other in (("W2", "X"), ("W2", "dY"), ("W1", "W1"), ("Wg", "W1"), ("W2", "W2")):
        with pytest.raises(ValueError, match="overlaps"):
            ff.dense_backward(desc, **t, grads={k: t[other]})
    with pytest.raises(ValueError, match="overlaps"):
        ff.dense_backward(desc, **t, dX=two, grads={"W2": two})
    both = torch.zeros(150, 64)
    with pytest.raises(ValueError, match="overlaps"):
        ff.dense_backward(desc, **dict(t, dY=both[:100]), dX=both[50:])
    # side by side is fine: the call gets as far as asking for a GPU
    with pytest.raises(ValueError, match="GPU"):
        ff.dense_backward(desc, **t, grads={"W1": flat[:6400].view(64, 100), "Wg": flat[6400:].view(64, 100), "W2": two})
    layers = [{k: torch.zeros_like(t[k]) for k in ("W1", "Wg", "W2")} for _ in range(2)]
    saved = torch.zeros(1 << 20, dtype=torch.uint8)
    for bad in (layers[0]["W2"], layers[1]["W2"], t["dY"]):
        grads = [{k: torch.zeros_like(W[k]) for k in W} for W in layers]
        grads[1]["W2"] = bad
        with pytest.raises(ValueError, match="overlaps"):
            ff.dense_stack_backward(desc, layers, saved, t["dY"], grads=grads)


def test_clipped_gradients_do_not_go_where_another_one_lies():
    a, b, c, one = torch.ones(8), torch.ones(8), torch.ones(8), torch.ones(1)
    for out in ([b, a], [b, c], [c, a]):
        with pytest.raises(ValueError, match="still read"):
            ff.grad_clip([a, b], one, 1.0, out=out)
        with pytest.raises(ValueError, match="still read"):
            ff.clip_grad_norm([a, b], 1.0, out=out)
    for out in ([a, c], [c, b], [a, b], None):          # in place, or elsewhere: as far as asking for a GPU
        with pytest.raises(ValueError, match="GPU"):
            ff.grad_clip([a, b], one, 1.0, out=out)
    e = torch.ones(8)[:0]
    with pytest.raises(ValueError, match="GPU"):
        ff.grad_clip([a, e, e], one, 1.0, out=[a, e, e])


def test_a_limit_that_is_not_a_number_is_refused():
    """A limit that a program computed to NaN would otherwise leave the gradients of a step unclipped."""
    desc = ff.make_desc(64, 100, "gelu", "f32")
    at = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: the calls fail validation, or have nothing to launch
    p = (ctypes.c_void_p * 1)(0x1000)

    def call(max_norm, layers=1):
        return ff.lib.ffsplit_dense_stack_backward(ctypes.byref(desc), layers, p, None, p, at, at, 4, 1e-6, p, None, p, 0, max_norm,
                                                   None, None, at, 1 << 40, None)

    assert call(math.nan) == -3 and call(math.nan, 0) == -3
    assert call(0.0, 0) == 0 and call(-1.0, 0) == 0 and call(math.inf, 0) == 0


def test_a_graph_does_not_end_in_a_call_unnoticed():
    """Tokens that require grad would give an output that does not; parameters as weights are the ordinary case."""
    desc, t = _layer(T=4, act="gelu")
    W1, W2 = torch.nn.Parameter(t["W1"]), torch.nn.Parameter(t["W2"])
    X = torch.zeros(4, 64, requires_grad=True)
    res, Y = torch.zeros(4, 64, requires_grad=True), torch.zeros(4, 64, requires_grad=True)
    for kw in (dict(X=X), dict(X=X * 2), dict(X=t["X"], residual=res, y_f32=True), dict(X=t["X"], Y=Y)):
        with pytest.raises(ValueError, match="requires grad"):
            ff.dense_forward(desc, W1=W1, Wg=None, W2=W2, **kw)
    with pytest.raises(ValueError, match="requires grad"):
        ff.dense_stack_forward(desc, [{"W1": W1, "W2": W2}], X * 2)
    # as far as asking for a GPU
    with pytest.raises(ValueError, match="GPU"):
        ff.dense_forward(desc, X.detach(), W1, None, W2)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        ff.dense_forward(desc, X, W1, None, W2)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        ff.dense_stack_forward(desc, [{"W1": W1, "W2": W2}], X)


def test_clipping_without_the_norm_is_refused():
    desc, t = _layer(T=4, act="gelu")
    saved = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="needs the norm"):
        ff.dense_stack_backward(desc, [{"W1": t["W1"], "W2": t["W2"]}], saved, t["dY"], max_norm=1.0, want_norm=False)


def test_layers_may_carry_more_than_their_weights():
    """A program's layer dicts hold other things as well: the stack's calls look at W1, Wg and W2."""
    desc, t = _layer(T=4, act="gelu")
    layers = [{"W1": t["W1"], "W2": t["W2"], "Wg": None, "name": "ffn.0", "steps": 3}]
    grads = [{"W1": torch.zeros_like(t["W1"]), "W2": torch.zeros_like(t["W2"])}]
    saved = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        ff.dense_stack_backward(desc, layers, saved, t["dY"], grads=grads)
