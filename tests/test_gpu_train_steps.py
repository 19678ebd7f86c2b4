"""Training steps of stacks as a program makes them: micro-batches, bf16 at ordinary widths."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import train_util as tu
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def ff():
    import paper_2401_04044_amd as m
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_micro_batches_take_the_norm_once(ff, dtype):
    """Three micro-batches accumulated in fp32, the norm and clipping with the last: the parts' gradients added, then clipped."""
    T, d, f, n = 40, 64, 203, 2
    rng = np.random.default_rng(50)
    desc = ff.make_desc(d, f, "swiglu", dtype)
    dev = [dict(zip(("W1", "Wg", "W2"), tu.to_dev(tu.make_layer(rng, d, f, True, T, dtype)[1:4], dtype))) for _ in range(n)]
    acc = [{k: torch.zeros(t.shape, device="cuda") for k, t in W.items()} for W in dev]
    total = [{k: torch.zeros(t.shape, device="cuda") for k, t in W.items()} for W in dev]
    for i in range(3):
        x, dy = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda")
        saved = ff.dense_stack_forward(desc, dev, x, want_saved=True)
        one, own_norm, flag = ff.dense_stack_backward(desc, dev, saved, dy.clone(), grad_f32=True)
        assert int(flag) == 0
        for t, o in zip(total, one):
            for k in t:
                t[k] += o[k]
        last = i == 2
        limit = 0.5 * float(torch.cat([t[k].double().flatten() for t in total for k in t]).norm()) if last else 0.0
        got, norm, flag = ff.dense_stack_backward(desc, dev, saved, dy.clone(), grads=acc, accumulate=True, grad_f32=True,
                                                  max_norm=limit, want_norm=last)
        assert got[0]["W1"] is acc[0]["W1"]
        if not last:
            assert norm is None and flag is None
            assert all(torch.equal(a[k], t[k]) for a, t in zip(acc, total) for k in t)
    want = ff.grad_clip([t[k] for t in total for k in t], norm, limit)
    assert int(flag) == 0 and abs(float(norm) - 2 * limit) <= 2.0 ** -22 * limit
    assert all(torch.equal(a, w) for a, w in zip([a[k] for a in acc for k in a], want))
