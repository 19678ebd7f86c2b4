"""The training path on more tokens than one launch has room for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    import paper_2401_04044_amd as m
    return m


@pytest.mark.parametrize("bf16", [True, False])
def test_the_norm_of_more_rows_than_a_launch_has_threads_for(ff, bf16):
    T, d = (1 << 24) + 3, 8
    kind = ff.BF16 if bf16 else ff.F32
    x = torch.randn(T, d, device="cuda")
    n = ff.token_rmsnorm(x, kind)
    for a, b in ((0, 1000), ((1 << 23) - 500, (1 << 23) + 500), (T - 1000, T)):
        assert torch.equal(n[a:b], ff.token_rmsnorm(x[a:b].contiguous(), kind))


def test_a_stack_trained_on_more_than_2_to_24_tokens(ff):
    """First and last tokens alone give the same stream and gradient; the weights' gradients are the sum of the parts'."""
    T, d, f = (1 << 24) + 21, 8, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    layers = [{"W1": torch.randn(d, f, generator=g, device="cuda").mul_(0.3).bfloat16(),
               "Wg": torch.randn(d, f, generator=g, device="cuda").mul_(0.3).bfloat16(),
               "W2": torch.randn(f, d, generator=g, device="cuda").mul_(0.3).bfloat16()}]
    x0, dy = torch.randn(T, d, generator=g, device="cuda"), torch.randn(T, d, generator=g, device="cuda")

    def go(a, b):
        x, dx = x0[a:b].clone(), dy[a:b].clone()
        saved = ff.dense_stack_forward(desc, layers, x, want_saved=True)
        grads, norm, flag = ff.dense_stack_backward(desc, layers, saved, dx, grad_f32=True)
        assert int(flag) == 0
        return x, dx, grads[0]

    x, dx, whole = go(0, T)
    cut = 1 << 23
    total = None
    for a, b in ((0, cut), (cut, T)):
        px, pdx, part = go(a, b)
        assert torch.equal(px, x[a:b]) and torch.equal(pdx, dx[a:b])
        total = part if total is None else {k: total[k] + part[k] for k in part}
    for k in whole:    # fp32 sums of 2^19 matrix instructions in other orders: 2^9.5 half steps as they add up at random
        assert float((total[k] - whole[k]).norm() / whole[k].norm()) < 2.0 ** -12, k


def test_the_norm_of_the_longest_row(ff):
    """The last columns of a row of 2^31 - 8: a 31-bit column index would have wrapped."""
    d = (1 << 31) - 8
    x = torch.ones(1, d, device="cuda")
    n = ff.token_rmsnorm(x)
    assert bool((n[:, -3000:] == 1).all()) and bool((n[:, ::4099] == 1).all())
