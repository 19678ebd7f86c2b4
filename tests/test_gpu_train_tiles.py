"""Every tile that the training path's products may take, whole and in ranges of the reduction, entry by entry against 64
bits: the sizes of train_sizes.py, which test_plain_plan.py compares with the choice."""
import numpy as np
import pytest
import torch

import train_ref as tr
from train_sizes import SIZES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    import paper_2401_04044_amd as m
    return m


def _check(ff, T, d, f, gated, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T + 3 * d + 7 * f)
    X, W1, Wg, W2, dY = tr.make_layer(gen, d, f, gated, T, dtype)
    desc = ff.make_desc(d, f, "swiglu" if gated else "gelu", dtype)
    kept = torch.full((ff.dense_kept_bytes(desc, T),), 0xFF, dtype=torch.uint8, device="cuda")
    ws = torch.full((max(ff.workspace_bytes(desc, c, T) for c in (ff.WS_DENSE_FORWARD, ff.WS_DENSE_BACKWARD)),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    Y, _ = ff.dense_forward(desc, X, W1, Wg, W2, saved=kept, workspace=ws)
    ws.fill_(0xFF)
    dX, wide = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, grad_f32=True, workspace=ws)
    names = ("W1", "Wg", "W2") if gated else ("W1", "W2")
    wide8 = [None if t is None else t.double() for t in (X, W1, Wg, W2, dY)]
    want, inner = tr.reference(*wide8)
    b = tr.bounds(*wide8, inner, dtype)
    del inner, wide8
    what = f"{dtype} T{T} d{d} f{f} {'gated' if gated else 'gelu'} "
    for name, got, u in [("Y", Y, tr.U[dtype]), ("dX", dX, tr.U[dtype])] + [(k, wide[k], tr.U["f32"]) for k in names]:
        tr.assert_within(got, want[name], b[name], u, what + name)
        # (bounds of long sums are wide: the whole must be as near as roundings that go either way leave it)
        if got.numel() >= 1024:
            e = float((got.double() - want[name]).norm() / want[name].norm())
            assert e < {"bf16": 1e-2, "f32": 1e-5}[dtype], (what + name, e)
    # in the storage type: the same sums, rounded once; accumulated: added in fp32 to what is there
    _, narrow = ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, want_dx=False)
    base = {k: torch.randn(wide[k].shape, generator=gen, device="cuda") * wide[k].std() for k in names if wide[k].numel() > 1}
    acc = {k: t.clone() for k, t in base.items()}
    ff.dense_backward(desc, X, W1, Wg, W2, kept, dY, want_dx=False, grads=acc, accumulate=True, grad_f32=True)
    for k in names:
        assert torch.equal(narrow[k], wide[k].to(narrow[k].dtype)), what + k
        if k in base:
            assert torch.equal(acc[k], wide[k] + base[k]), what + k


@pytest.mark.parametrize("T,d,f,gated,dtype", SIZES)
def test_every_tile_entry_by_entry(ff, T, d, f, gated, dtype):
    _check(ff, T, d, f, gated, dtype)


# a Llama-2-7B-sized layer on a ragged batch: six products of 256x256 tiles over many slabs, with a partial tile at every edge
@pytest.mark.parametrize("T,d,f,gated,dtype", [(1100, 4096, 11008, True, "bf16"), (2000, 4096, 550, True, "bf16"), (410, 696, 2403, True, "f32"),
                                               (689, 336, 1455, False, "f32")])
def test_ordinary_layers_entry_by_entry(ff, T, d, f, gated, dtype):
    _check(ff, T, d, f, gated, dtype)
