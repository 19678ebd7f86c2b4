"""The training path on the GPU against the fp64 oracle: entry by entry within what its roundings allow (train_util)."""
import math

import numpy as np
import pytest
import torch

import gpu_util as gu
import train_util as tu
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu
EPS = 1e-6
TDT = gu.TDT


@pytest.fixture(scope="module")
def ff():
    import paper_2401_04044_amd as m
    return m


def _guarded(n, device="cuda"):
    return gu.Guarded(n, device)


def _run_layer(ff, desc, host, dtype, **kw):
    """Forward keeping what the backward needs, backward; buffers between sentinels."""
    X, W1, Wg, W2, dY = tu.to_dev(host, dtype)
    T = X.shape[0]
    kept = _guarded(ff.dense_kept_bytes(desc, T))
    w1, w2 = _guarded(ff.workspace_bytes(desc, ff.WS_DENSE_FORWARD, T)), _guarded(ff.workspace_bytes(desc, ff.WS_DENSE_BACKWARD, T))
    Y, _ = ff.dense_forward(desc, X, W1, Wg, W2, saved=kept.view, workspace=w1.view)
    dX, g = ff.dense_backward(desc, X, W1, Wg, W2, kept.view, dY, workspace=w2.view, **kw)
    for b, what in ((kept, "kept"), (w1, "forward scratch"), (w2, "backward scratch")):
        b.check(what)
    return Y, dX, g


def _check_layer(ff, T, d, f, gated, dtype, seed=0, **kw):
    rng = np.random.default_rng(1000 * T + 10 * f + d + seed)
    host = tu.make_layer(rng, d, f, gated, T, dtype)
    X, W1, Wg, W2, dY = host
    desc = ff.make_desc(d, f, "swiglu" if gated else "gelu", dtype)
    Y, dX, g = _run_layer(ff, desc, host, dtype, **kw)
    want, kept = orc.dense_forward(X, W1, Wg, W2)
    wdX, wg = orc.dense_backward(X, W1, Wg, W2, kept, dY)
    u_grad = tu.U["f32"] if kw.get("grad_f32") else tu.U[dtype]
    b = tu.dense_bounds(X, W1, Wg, W2, kept, dY, tu.U[dtype], u_grad)
    what = f"{dtype} T{T} d{d} f{f} {'gated' if gated else 'gelu'} "
    for name, got, ref in [("Y", Y, want), ("dX", dX, wdX)] + [(k, g[k], wg[k]) for k in ("W1", "Wg", "W2") if wg[k] is not None]:
        tu.assert_within(gu.host(got), ref, b[name], what + name)
        # (one column of a few tokens can cancel to nothing; the whole tensor cannot)
        if T >= 16 and f >= 16:
            e = gu.relf(gu.host(got), ref)
            assert e < gu.TOL[dtype], (what + name, e)
    assert gated or g["Wg"] is None


# one token, a few, tile edges and beyond; widths below a tile, odd, aligned, more than one tile; reductions
# shorter than a slab and with remainders
SHAPES = [(1, 8, 1), (32, 200, 300), (31, 136, 2050), (1, 264, 1000), (2, 64, 7), (3, 136, 130), (16, 64, 64), (17, 72, 129), (33, 520, 96), (64, 128, 256),
          (65, 256, 550), (129, 136, 257), (200, 264, 1003), (300, 512, 640)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,d,f", SHAPES)
def test_layer_forward_and_gradients(ff, T, d, f, gated, dtype):
    _check_layer(ff, T, d, f, gated, dtype)


@pytest.mark.parametrize("T,d,f,gated", [(1030, 1024, 2816, True), (2048, 768, 1800, False), (700, 2048, 1024, True)])
def test_layer_with_large_tiles(ff, T, d, f, gated):
    _check_layer(ff, T, d, f, gated, "bf16")


@pytest.mark.parametrize("T", [20, 70])           # (up to 32 tokens the bf16 gradients have a kernel of their own)
@pytest.mark.parametrize("dtype,f", [("bf16", 96), ("bf16", 99), ("f32", 99)])
def test_gradients_in_fp32_and_accumulated(ff, dtype, f, T):
    d = 64
    _check_layer(ff, T, d, f, True, dtype, grad_f32=True)
    rng = np.random.default_rng(8)
    host = tu.make_layer(rng, d, f, True, T, dtype)
    desc = ff.make_desc(d, f, "swiglu", dtype)
    X, W1, Wg, W2, dY = tu.to_dev(host, dtype)
    _, kept = ff.dense_forward(desc, X, W1, Wg, W2, want_saved=True)
    _, once = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, grad_f32=True)
    acc = {k: g.clone() for k, g in once.items()}
    ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, grads=acc, accumulate=True, grad_f32=True)
    for k in once:      # twice the same sum: one rounding of x + x, which is exact
        assert torch.equal(acc[k], 2 * once[k]), k
    # in the storage type: the sum is formed in fp32 from what the buffer holds and rounded once
    base = {k: (torch.randn_like(g) * g.std()).to(TDT[dtype]) for k, g in once.items()}
    got = {k: g.clone() for k, g in base.items()}
    ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, grads=got, accumulate=True)
    for k in once:
        assert torch.equal(got[k], (once[k] + base[k].float()).to(TDT[dtype])), k


def test_parts_of_the_backward_alone_equal_the_whole(ff):
    T, d, f = 50, 64, 99
    host = tu.make_layer(np.random.default_rng(2), d, f, True, T, "bf16")
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    X, W1, Wg, W2, dY = tu.to_dev(host, "bf16")
    Y, kept = ff.dense_forward(desc, X, W1, Wg, W2, want_saved=True)
    before = kept.clone()
    assert torch.equal(Y, ff.dense_forward(desc, X, W1, Wg, W2))
    dX, g = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY)
    again, _ = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, grads={})
    assert torch.equal(dX, again)
    for k in g:
        none, one = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, want_dx=False, grads={k: torch.empty_like(g[k])})
        assert none is None and torch.equal(one[k], g[k]), k
    assert torch.equal(kept, before)


def test_residual_and_fp32_output(ff):
    T, d, f = 70, 64, 200
    host = tu.make_layer(np.random.default_rng(3), d, f, True, T, "bf16")
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    X, W1, Wg, W2, _ = tu.to_dev(host, "bf16")
    res = torch.randn(T, d, device="cuda")
    plain = ff.dense_forward(desc, X, W1, Wg, W2, y_f32=True)
    assert torch.equal(plain.bfloat16(), ff.dense_forward(desc, X, W1, Wg, W2))
    want = plain + res
    assert torch.equal(ff.dense_forward(desc, X, W1, Wg, W2, residual=res, y_f32=True), want)
    assert torch.equal(ff.dense_forward(desc, X, W1, Wg, W2, residual=res), want.bfloat16())
    x = res.clone()
    assert torch.equal(ff.dense_forward(desc, X, W1, Wg, W2, Y=x, residual=x, y_f32=True), want)


@pytest.mark.parametrize("T", [1, 5, 70])
def test_a_bad_token_stays_alone(ff, T):
    """Infinities and NaN in one token reach only that token's output and gradient (and the weights' gradients)."""
    d, f = 64, 99
    host = tu.make_layer(np.random.default_rng(4), d, f, True, T, "bf16")
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    X, W1, Wg, W2, dY = tu.to_dev(host, "bf16")
    Y, kept = ff.dense_forward(desc, X, W1, Wg, W2, want_saved=True)
    dX, _ = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY)
    for value in (float("nan"), float("inf")):
        Xb = X.clone()
        Xb[T // 2, 3] = value
        Yb, keptb = ff.dense_forward(desc, Xb, W1, Wg, W2, want_saved=True)
        dXb, gb = ff.dense_backward(desc, Xb, W1, Wg, W2, keptb, dY)
        rest = [t for t in range(T) if t != T // 2]
        assert not torch.isfinite(Yb[T // 2]).all()
        assert torch.equal(Yb[rest], Y[rest]) and torch.equal(dXb[rest], dX[rest])
        assert not torch.isfinite(gb["W2"]).all()


def test_a_factor_beyond_fp16_is_not_hidden(ff):
    """A kept derivative beyond 65504 makes the gradients behind it non-finite; one below it does not."""
    T, d, f = 4, 64, 40
    host = tu.make_layer(np.random.default_rng(14), d, f, True, T, "bf16")
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    X, W1, Wg, W2, dY = tu.to_dev(host, "bf16")
    for scale, fine in ((512.0, True), (1e7, False)):     # |z| of some tens, of some hundred thousand
        Y, kept = ff.dense_forward(desc, X * scale, W1, Wg, W2, want_saved=True)
        assert torch.isfinite(Y).all()
        dX, g = ff.dense_backward(desc, X * scale, W1, Wg, W2, kept, dY)
        _, flag = ff.grad_norm([g["W1"], g["Wg"]])
        assert (int(flag) == 0) == fine and bool(torch.isfinite(dX).all()) == fine


def test_memory_around_the_operands_is_not_used(ff):
    """Rows behind the last and in front of the first are NaN: nothing of them reaches a result, nothing is written there."""
    T, d, f = 37, 72, 101
    for dtype in ("bf16", "f32"):
        host = tu.make_layer(np.random.default_rng(5), d, f, True, T, dtype)
        desc = ff.make_desc(d, f, "swiglu", dtype)
        plain = tu.to_dev(host, dtype)
        _, kept = ff.dense_forward(desc, *plain[:4], want_saved=True)
        want = [ff.dense_forward(desc, *plain[:4])] + list(ff.dense_backward(desc, *plain[:4], kept, plain[4]))
        pad = 4096

        def fenced(t):
            buf = torch.full((t.numel() + 2 * pad,), float("nan"), dtype=t.dtype, device="cuda")
            buf[pad:pad + t.numel()] = t.reshape(-1)
            return buf, buf[pad:pad + t.numel()].view(t.shape)

        bufs, ins = zip(*[fenced(t) for t in plain])
        outs = [fenced(torch.zeros_like(t)) for t in (want[0], want[1], want[2]["W1"], want[2]["Wg"], want[2]["W2"])]
        _, kept = ff.dense_forward(desc, *ins[:4], Y=outs[0][1], want_saved=True)
        ff.dense_backward(desc, *ins[:4], kept, ins[4], dX=outs[1][1],
                          grads={"W1": outs[2][1], "Wg": outs[3][1], "W2": outs[4][1]})
        flat = [want[0], want[1], want[2]["W1"], want[2]["Wg"], want[2]["W2"]]
        for (buf, got), ref in zip(outs, flat):
            assert torch.equal(got, ref)
        for buf in list(bufs) + [o[0] for o in outs]:
            assert torch.isnan(buf[:pad]).all() and torch.isnan(buf[-pad:]).all()


@pytest.mark.parametrize("T,d,f", [(1, 72, 99), (31, 200, 1500), (32, 1000, 300), (33, 264, 131), (47, 72, 2050), (100, 136, 37)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_buffers_may_hold_anything(ff, T, d, f, dtype):
    """Scratch and kept state full of NaN patterns before the call: the same bits as with zeros."""
    host = tu.make_layer(np.random.default_rng(T), d, f, True, T, dtype)
    desc = ff.make_desc(d, f, "swiglu", dtype)
    X, W1, Wg, W2, dY = tu.to_dev(host, dtype)

    def go(byte):
        kept = torch.full((ff.dense_kept_bytes(desc, T),), byte, dtype=torch.uint8, device="cuda")
        w1 = torch.full((ff.workspace_bytes(desc, ff.WS_DENSE_FORWARD, T),), byte, dtype=torch.uint8, device="cuda")
        w2 = torch.full((ff.workspace_bytes(desc, ff.WS_DENSE_BACKWARD, T),), byte, dtype=torch.uint8, device="cuda")
        alone = ff.dense_forward(desc, X, W1, Wg, W2, workspace=w1)
        w1.fill_(byte)
        Y = ff.dense_forward(desc, X, W1, Wg, W2, saved=kept, workspace=w1)[0]
        dX, g = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, workspace=w2)
        return [alone, Y, dX, g["W1"], g["Wg"], g["W2"]]

    for a, b in zip(go(0), go(0xFF)):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("T", [3, 40])
def test_weights_beyond_two_gib(ff, T):
    """Offsets into the weights pass 32 bits, along either axis of them."""
    d, f = 8192, 139_264
    assert d * f * 2 > 1 << 31
    g = torch.Generator(device="cuda")
    g.manual_seed(2)

    def normal(shape, std):
        out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        for part in out.split(max(1, (1 << 27) // shape[1])):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(std))
        return out

    W1, W2 = normal((d, f), 0.01), normal((f, d), 0.01)
    X, dY = normal((T, d), 1.0), normal((T, d), 1.0)
    desc = ff.make_desc(d, f, "gelu", "bf16")
    Y, kept = ff.dense_forward(desc, X, W1, None, W2, want_saved=True)
    dX, dW = ff.dense_backward(desc, X, W1, None, W2, kept, dY)
    want_Y, want_dX = torch.zeros(T, d, device="cuda"), torch.zeros(T, d, device="cuda")
    x, dy, step = X.float(), dY.float(), 8704
    for a in range(0, f, step):
        w1, w2 = W1[:, a:a + step].float(), W2[a:a + step].float()
        z = (x @ w1).double()
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        H, D = (z * cdf).float(), (cdf + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)).float()
        want_Y += H @ w2
        dU = (dy @ w2.t()) * D
        want_dX += dU @ w1.t()
        if a in (0, f - step):
            for got, ref in ((dW["W1"][:, a:a + step], x.t() @ dU), (dW["W2"][a:a + step], H.t() @ dy)):
                assert float((got.float() - ref).norm() / ref.norm()) < gu.TOL["bf16"]
    for got, ref in ((Y, want_Y), (dX, want_dX)):
        assert float((got.float() - ref).norm() / ref.norm()) < gu.TOL["bf16"]


def test_no_tokens(ff):
    d, f = 64, 99
    for dtype in ("bf16", "f32"):
        desc = ff.make_desc(d, f, "swiglu", dtype)
        _, W1, Wg, W2, _ = tu.to_dev(tu.make_layer(np.random.default_rng(6), d, f, True, 1, dtype), dtype)
        X = torch.empty(0, d, dtype=TDT[dtype], device="cuda")
        Y, kept = ff.dense_forward(desc, X, W1, Wg, W2, want_saved=True)
        assert Y.shape == (0, d)
        dX, g = ff.dense_backward(desc, X, W1, Wg, W2, kept, X)
        assert dX.shape == (0, d) and all((g[k] == 0).all() for k in g)
        ones = {k: torch.ones_like(g[k]) for k in g}
        ff.dense_backward(desc, X, W1, Wg, W2, kept, X, grads=ones, accumulate=True)
        assert all((ones[k] == 1).all() for k in ones)


# ---------------------------------------------------------------- the norm

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 8), (5, 64), (33, 768), (7, 2048), (6, 2056), (9, 5120), (3, 8192), (4, 8200), (2, 20000)])
def test_rmsnorm_backward(ff, T, d, dtype):
    rng = np.random.default_rng(T + d)
    x = (rng.standard_normal((T, d)) * np.exp(rng.uniform(-6, 6, (T, 1)))).astype(np.float32)
    if T > 2:
        x[2] = 0.0                                # r = eps^-1/2
    dn = gu.dev(rng.standard_normal((T, d)), dtype)
    res = rng.standard_normal((T, d)).astype(np.float32)
    xd, rd = torch.from_numpy(x).cuda(), torch.from_numpy(res).cuda()
    r = 1 / np.sqrt((x.astype(np.float64) ** 2).mean(1, keepdims=True) + EPS)
    dnh = gu.host(dn)
    # fp32 sums of d terms; each term of the result a few roundings
    m = np.abs(r * dnh) + np.abs(x) * r ** 3 * (np.abs(x) * np.abs(dnh)).mean(1, keepdims=True)
    for residual in (None, res):
        want = orc.token_rmsnorm_backward(x, dnh, EPS, residual)
        bound = (2 * tu.g(d) + 8 * 2.0 ** -24) * m + (0 if residual is None else 2.0 ** -24 * np.abs(residual))
        dx, cast = ff.token_rmsnorm_backward(xd, dn, EPS, None if residual is None else rd, want_cast=True)
        tu.assert_within(gu.host(dx), want, (bound, tu.U["f32"]), f"rmsnorm backward {T} {d}")
        assert torch.equal(cast, dx.to(dn.dtype))
    acc = rd.clone()                              # the residual's gradient in place
    ff.token_rmsnorm_backward(xd, dn, EPS, residual=acc, dx=acc)
    assert torch.equal(acc, dx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(5, 520), (6, 1016), (3, 1024), (5, 1032), (3, 1536)])
def test_rmsnorm_backward_by_wavefront_and_by_workgroup(ff, T, d, dtype):
    test_rmsnorm_backward(ff, T, d, dtype)


def test_rmsnorm_backward_of_many_rows(ff):
    """More rows than one launch has workgroups: every row is the one that a short call gives."""
    T, d = (1 << 22) + 5, 8
    x = torch.randn(T, d, device="cuda")
    dn = torch.randn(T, d, device="cuda")
    dx = ff.token_rmsnorm_backward(x, dn, EPS)
    for a, b in ((0, 1000), (T - 1000, T)):
        assert torch.equal(dx[a:b], ff.token_rmsnorm_backward(x[a:b].contiguous(), dn[a:b].contiguous(), EPS))
    assert ff.token_rmsnorm_backward(x[:0], dn[:0], EPS).shape == (0, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("T,d,f", [(3, 64, 1), (9, 72, 2047), (33, 136, 4103)])
def test_rows_that_are_padded(ff, T, d, f, gated, dtype):
    """d_ff not a multiple of 8: the weights' copies with aligned rows, one word of a row to several passes of a workgroup."""
    test_layer_forward_and_gradients(ff, T, d, f, gated, dtype)


# ---------------------------------------------------------------- norm over all gradients, clipping

def _grads(rng, sizes, dtypes):
    return [gu.dev(rng.standard_normal(n).astype(np.float32), t) for n, t in zip(sizes, dtypes)]


@pytest.mark.parametrize("sizes", [[1], [7], [0, 5, 0], [16384], [16385, 3], [40000, 1, 8192, 123457], [33] * 57, [9] * 300, []])
@pytest.mark.parametrize("mixed", [False, True])
def test_grad_norm_and_clip(ff, sizes, mixed):
    rng = np.random.default_rng(len(sizes) + sum(sizes))
    dts = ["bf16" if mixed and i % 2 == 0 else "f32" for i in range(len(sizes))]
    grads = _grads(rng, sizes, dts)
    before = [g.clone() for g in grads]
    want = orc.grad_norm([gu.host(g) for g in grads])
    norm, flag = ff.grad_norm(grads)
    # squares and sums in 64 bits: one rounding to fp32
    assert abs(float(norm) - want) <= 2.0 ** -24 * want + 1e-300 and int(flag) == 0
    if want == 0:
        return
    for limit in (0.3 * want, 2 * want, math.inf):
        out = [torch.empty_like(g) for g in grads]
        clipped = ff.grad_clip(grads, norm, limit, out=out)
        for g, b, o, dt in zip(grads, before, clipped, dts):
            assert torch.equal(g, b)
            if limit > want:
                assert torch.equal(o, b)
            else:       # one fp32 rounding of the factor (half a step, and one of the division's), one of the product
                ref = gu.host(b) * (np.float32(limit) / want)
                assert (np.abs(gu.host(o) - ref) <= (3 * 2.0 ** -24 + tu.U[dt]) * np.abs(ref)).all()
    n2, f2, same = ff.clip_grad_norm(grads, 0.3 * want)
    assert same is grads and torch.equal(n2, norm) and int(f2) == 0
    ref = ff.grad_clip(before, norm, 0.3 * want, out=[torch.empty_like(g) for g in grads])
    assert all(torch.equal(a, b) for a, b in zip(grads, ref))


def test_grad_norm_at_the_ends_of_the_range(ff):
    big = torch.full((4096,), 3e38, device="cuda")              # the norm is beyond fp32
    norm, flag = ff.grad_norm([big])
    assert math.isinf(float(norm)) and int(flag) == ff.E_NONFINITE
    huge = torch.full((1024,), 1e30, dtype=torch.bfloat16, device="cuda")     # its squares are
    norm, flag = ff.grad_norm([huge])
    assert abs(float(norm) / (32 * float(huge[0])) - 1) < 2.0 ** -23 and int(flag) == 0
    tiny = torch.full((1024,), 1e-30, device="cuda")
    norm, _ = ff.grad_norm([tiny])
    assert abs(float(norm) / (32 * float(tiny[0])) - 1) < 2.0 ** -23
    for bad in (float("nan"), float("inf"), float("-inf")):
        g = [torch.ones(5000, dtype=torch.bfloat16, device="cuda"), torch.ones(77, device="cuda")]
        g[0][4999] = bad
        before = [t.clone() for t in g]
        norm, flag, out = ff.clip_grad_norm(g, 0.5)
        assert int(flag) == ff.E_NONFINITE and not math.isfinite(float(norm))
        assert all(torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32),
                               b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32)) for a, b in zip(out, before))


def test_grad_clip_writes_nothing_else(ff):
    buf = torch.full((1000,), 7.0, device="cuda")
    g = buf[64:64 + 333]
    ff.clip_grad_norm([g], 1.0)
    assert (buf[:64] == 7).all() and (buf[64 + 333:] == 7).all() and abs(float(g.norm()) - 1) < 1e-5


# ---------------------------------------------------------------- all of them together

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [True, False])
def test_stack_step(ff, gated, dtype):
    """Three layers: forward, backward, clipping, against the oracle's chain."""
    T, d, f, n = 37, 72, 203, 3
    rng = np.random.default_rng(9)
    hosts = [tu.make_layer(rng, d, f, gated, T, dtype) for _ in range(n)]
    layers = [(h[1], h[2], h[3]) for h in hosts]
    x0, dy = hosts[0][0], rng.standard_normal((T, d)).astype(np.float32)
    desc = ff.make_desc(d, f, "swiglu" if gated else "gelu", dtype)
    dev = [dict(zip(("W1", "Wg", "W2"), tu.to_dev(W, dtype))) for W in layers]
    x, dx = torch.from_numpy(x0).cuda(), torch.from_numpy(dy).cuda()
    only = ff.dense_stack_forward(desc, dev, x.clone())
    saved = ff.dense_stack_forward(desc, dev, x, want_saved=True)
    assert torch.equal(only, x)
    again = dx.clone()
    free, norm, flag = ff.dense_stack_backward(desc, dev, saved, again)
    wx, tape = orc.stack_forward(layers, x0, EPS)
    wdx, wg = orc.stack_backward(layers, tape, dy, EPS)
    # every layer's roundings pass through the layers behind: a few times one layer's bar
    tol = {"bf16": 3e-2, "f32": 1e-5}[dtype]
    assert gu.relf(gu.host(x), wx) < tol and gu.relf(gu.host(again), wdx) < tol
    names = ("W1", "Wg", "W2") if gated else ("W1", "W2")
    for l in range(n):
        for k in names:
            assert gu.relf(gu.host(free[l][k]), wg[l][k]) < tol, (l, k)
        assert gated or free[l]["Wg"] is None
    # the norm is that of the gradients returned, and clipping scales those
    flat = [free[l][k] for l in range(n) for k in names]
    own = orc.grad_norm([gu.host(t) for t in flat])
    assert abs(float(norm) - own) <= 2.0 ** -23 * own and int(flag) == 0
    dx2 = dx.clone()
    clipped, norm2, _ = ff.dense_stack_backward(desc, dev, saved, dx2, max_norm=0.5 * own)
    assert torch.equal(dx2, again) and torch.equal(norm2, norm)
    want = ff.grad_clip(flat, norm, 0.5 * own, out=[torch.empty_like(t) for t in flat])
    assert all(torch.equal(a, b) for a, b in zip([clipped[l][k] for l in range(n) for k in names], want))


def test_stack_is_its_parts(ff):
    """The driver gives what the single calls give, bit for bit."""
    T, d, f, n = 20, 64, 136, 2
    rng = np.random.default_rng(10)
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    hosts = [tu.make_layer(rng, d, f, True, T, "bf16") for _ in range(n)]
    dev = [dict(zip(("W1", "Wg", "W2"), tu.to_dev(h[1:4], "bf16"))) for h in hosts]
    x0, dy = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda")
    x, dx = x0.clone(), dy.clone()
    saved = ff.dense_stack_forward(desc, dev, x, want_saved=True)
    grads, _, _ = ff.dense_stack_backward(desc, dev, saved, dx)
    y, tape = x0.clone(), []
    for W in dev:
        m = ff.token_rmsnorm(y)
        out, kept = ff.dense_forward(desc, m, W["W1"], W["Wg"], W["W2"], residual=y, y_f32=True, want_saved=True)
        tape.append((y, m, kept))
        y = out
    assert torch.equal(x, y)
    g = dy.clone()
    for l in (1, 0):
        W, (xi, m, kept) = dev[l], tape[l]
        dn, dW = ff.dense_backward(desc, m, W["W1"], W["Wg"], W["W2"], kept, g.bfloat16())
        assert all(torch.equal(dW[k], grads[l][k]) for k in dW)
        g = ff.token_rmsnorm_backward(xi, dn, residual=g)
    assert torch.equal(dx, g)


def test_stack_accumulates_and_takes_no_tokens(ff):
    T, d, f, n = 9, 64, 40, 2
    rng = np.random.default_rng(11)
    desc = ff.make_desc(d, f, "gelu", "bf16")
    dev = [dict(zip(("W1", "Wg", "W2"), tu.to_dev(tu.make_layer(rng, d, f, False, T, "bf16")[1:4], "bf16"))) for _ in range(n)]
    x, dy = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda")
    saved = ff.dense_stack_forward(desc, dev, x, want_saved=True)
    once, norm, _ = ff.dense_stack_backward(desc, dev, saved, dy.clone(), grad_f32=True)
    acc = [{k: None if t is None else t.clone() for k, t in g.items()} for g in once]
    _, norm2, _ = ff.dense_stack_backward(desc, dev, saved, dy.clone(), grads=acc, accumulate=True, grad_f32=True)
    assert all(torch.equal(a[k], 2 * o[k]) for a, o in zip(acc, once) for k in ("W1", "W2"))
    assert abs(float(norm2) - 2 * float(norm)) <= 2.0 ** -22 * float(norm2)
    e = torch.empty(0, d, device="cuda")
    saved = ff.dense_stack_forward(desc, dev, e, want_saved=True)
    g, norm, flag = ff.dense_stack_backward(desc, dev, saved, e, max_norm=1.0)
    assert all((q[k] == 0).all() for q in g for k in ("W1", "W2")) and float(norm) == 0 and int(flag) == 0


# ---------------------------------------------------------------- streams, graphs, large offsets

def _step(ff, desc, dev, x, dx, saved, grads, ws):
    ff.dense_stack_forward(desc, dev, x, saved=saved, workspace=ws)
    return ff.dense_stack_backward(desc, dev, saved, dx, grads=grads, max_norm=0.1, workspace=ws)


@pytest.mark.parametrize("T", [1, 40, 300])
def test_captured_step_replays(ff, T):
    d, f, n = 128, 300, 2
    rng = np.random.default_rng(12)
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    dev = [dict(zip(("W1", "Wg", "W2"), tu.to_dev(tu.make_layer(rng, d, f, True, 1, "bf16")[1:4], "bf16"))) for _ in range(n)]
    ws = torch.empty(max(ff.workspace_bytes(desc, ff.WS_DENSE_STACK, T), 1 << 16), dtype=torch.uint8, device="cuda")
    saved = torch.empty(int(ff.lib.ffsplit_dense_stack_kept_bytes(desc, n, T)), dtype=torch.uint8, device="cuda")
    x, dx = torch.zeros(T, d, device="cuda"), torch.zeros(T, d, device="cuda")
    grads = [{k: torch.zeros_like(W[k]) for k in W} for W in dev]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(ff, desc, dev, x, dx, saved, grads, ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, norm, _ = _step(ff, desc, dev, x, dx, saved, grads, ws)
    for it in range(4):
        x0, dy = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda")
        ex, edx = x0.clone(), dy.clone()
        eg, en, _ = _step(ff, desc, dev, ex, edx, torch.empty_like(saved), None, torch.empty_like(ws))
        ws.fill_(0xFF)                           # nothing in the scratch has to be in any state
        x.copy_(x0)
        dx.copy_(dy)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, ex) and torch.equal(dx, edx) and torch.equal(norm, en), it
        assert all(torch.equal(a[k], b[k]) for a, b in zip(grads, eg) for k in a), it


def test_two_streams_at_once(ff):
    T, d, f = 200, 256, 700
    desc = ff.make_desc(d, f, "swiglu", "bf16")
    sets = [tu.to_dev(tu.make_layer(np.random.default_rng(s), d, f, True, T, "bf16"), "bf16") for s in (20, 21)]

    def go(t):
        Y, kept = ff.dense_forward(desc, *t[:4], want_saved=True)
        dX, g = ff.dense_backward(desc, *t[:4], kept, t[4])
        return [Y, dX, g["W1"], g["Wg"], g["W2"]]

    want = [go(t) for t in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for t, s in zip(sets, streams):
            with torch.cuda.stream(s):
                got.append(go(t))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_activations_beyond_four_gib(ff):
    """Offsets of H, D and dU pass 32 bits; first and last tokens alone give the same, and the weights' gradients
    are the sum of the halves' (fp32 sums in another order)."""
    d, f, T = 64, 16384, 140_000
    assert T * f * 2 > 1 << 32
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    dY = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    W1, Wg = (torch.randn(d, f, generator=g, device="cuda").mul_(0.125).bfloat16() for _ in range(2))
    W2 = torch.randn(f, d, generator=g, device="cuda").mul_(0.01).bfloat16()
    desc = ff.make_desc(d, f, "swiglu", "bf16")

    def go(a, b):
        x, dy = X[a:b].contiguous(), dY[a:b].contiguous()
        Y, kept = ff.dense_forward(desc, x, W1, Wg, W2, want_saved=True)
        return (Y,) + ff.dense_backward(desc, x, W1, Wg, W2, kept, dy, grad_f32=True)

    Y, dX, dW = go(0, T)
    cut = 70_016
    total = None
    for a, b in ((0, cut), (cut, T)):
        y, dx, dw = go(a, b)
        # (a shorter batch may sum in other ranges: half a step of bf16 on either side)
        for got, ref in ((y, Y[a:b]), (dx, dX[a:b])):
            assert float((got.float() - ref.float()).norm() / ref.float().norm()) < 2.0 ** -8
        total = dw if total is None else {k: total[k] + dw[k] for k in dw}
    for k in dW:
        assert float((total[k] - dW[k]).norm() / dW[k].norm()) < 1e-4, k
    sub = list(range(T - 50, T))
    want, kept = orc.dense_forward(gu.host(X[sub]), gu.host(W1), gu.host(Wg), gu.host(W2))
    wdx, _ = orc.dense_backward(gu.host(X[sub]), gu.host(W1), gu.host(Wg), gu.host(W2), kept, gu.host(dY[sub]))
    assert gu.relf(gu.host(Y[sub]), want) < gu.TOL["bf16"] and gu.relf(gu.host(dX[sub]), wdx) < gu.TOL["bf16"]


def test_results_repeat(ff):
    host = tu.make_layer(np.random.default_rng(30), 256, 999, True, 333, "bf16")
    desc = ff.make_desc(256, 999, "swiglu", "bf16")
    one, two = (_run_layer(ff, desc, host, "bf16") for _ in range(2))
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1]) and all(torch.equal(one[2][k], two[2][k]) for k in one[2])
