"""The choice of tile and ranges for the training path's products (host arithmetic, compiled here for the CPU): what the
GPU tests' sizes make it choose, and that no choice needs more than it may."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from train_sizes import SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
T128x128, T256x256, T64x64, T256x128 = range(4)
TILE = {T128x128: (128, 128), T256x256: (256, 256), T64x64: (64, 64), T256x128: (256, 128)}
RING = {T128x128: 5, T256x256: 4, T64x64: 8, T256x128: 4}       # stages
UP, DOWN, GRAD, DX, DUP, DDOWN = range(6)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text('#include "plain_plan.h"\n'
                   'extern "C" void plan(int which, long T, int d, int f, int planes, int bf16, long* out) {\n'
                   '  const auto s = ffsplit::dense_product(which, T, d, f, planes);\n'
                   '  const auto p = ffsplit::plain_plan(s, bf16);\n'
                   '  out[0] = p.shape; out[1] = p.split; out[2] = s.M; out[3] = s.N; out[4] = s.K; out[5] = s.segs;\n'
                   '  out[6] = s.twin || s.epi == ffsplit::EPI_GLU ? 2 : 1; }\n'
                   'extern "C" size_t room() { return ffsplit::PLAIN_PART_ROOM; }\n'
                   'extern "C" size_t bytes(int which, long T, int d, int f, int planes, int bf16) {\n'
                   '  return ffsplit::plain_part_bytes(ffsplit::dense_product(which, T, d, f, planes), bf16); }\n')
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-shared", "-fPIC",
                           "-I" + os.path.join(ROOT, "paper_2401_04044_amd", "csrc"), str(src), "-o", str(so)])
    lib = ctypes.CDLL(str(so))
    lib.plan.argtypes = [ctypes.c_int, ctypes.c_long] + [ctypes.c_int] * 4 + [ctypes.POINTER(ctypes.c_long)]
    lib.room.restype = ctypes.c_size_t
    lib.bytes.argtypes, lib.bytes.restype = [ctypes.c_int, ctypes.c_long] + [ctypes.c_int] * 4, ctypes.c_size_t

    def get(which, T, d, f, planes, bf16):
        out = (ctypes.c_long * 7)()
        lib.plan(which, T, d, f, planes, bf16, out)
        return list(out)

    get.room, get.bytes = lib.room(), lib.bytes
    return get


def _kinds(plan, T, d, f, gated, dtype):
    """Which kernels, of which kind of work, the products of a layer take."""
    bf16, out = dtype == "bf16", set()
    for which in range(6):
        planes = 1 + gated
        shape, split, _, _, K, segs, _ = plan(which, T, d, f, planes, bf16)
        if bf16 and which in (DUP, DDOWN) and K <= 32 and split == 1:
            shape = "walk"                    # (one slab, by workgroups that walk over the tiles)
        if which == DDOWN:
            planes = 0                        # the same product either way
        out.add((dtype, which, planes, shape, "ranges" if split > 1 else "whole"))
        out.add((dtype, which, shape, "aligned" if f % 8 == 0 else "not aligned"))
        if shape != "walk" and segs * -(-K // (32 if bf16 else 16)) // split >= 2 * RING[shape] + 3:
            out.add((dtype, which, planes, shape, "the ring wraps"))
    return out


def _sizes(rng, n):
    for _ in range(n):
        T, d, f = int(np.exp(rng.uniform(0, np.log(9000)))), 8 * int(np.exp(rng.uniform(0, np.log(768)))), int(np.exp(rng.uniform(0, np.log(12000))))
        yield T, d, (f + 7) // 8 * 8 if rng.random() < 0.3 else f, bool(rng.integers(2)), "bf16" if rng.random() < 0.6 else "f32"


def test_the_gpu_tests_reach_every_choice(plan):
    """Every tile of every product, whole and in ranges, that 40000 layers of up to 9000 tokens and 6144 x 12000 choose."""
    reached = set().union(*[_kinds(plan, *s) for s in SIZES])
    missing = {}
    for s in _sizes(np.random.default_rng(11), 40000):
        for k in _kinds(plan, *s) - reached:
            missing.setdefault(k, s)
    assert not missing, missing
    for dtype, tiles in (("bf16", (T128x128, T256x256, T64x64, T256x128)), ("f32", (T128x128, T64x64))):
        for which in range(6):
            for shape in tiles:
                assert any(k[:2] == (dtype, which) and shape in k[2:4] for k in reached), (dtype, which, shape)


def test_ranges_fit_their_scratch_and_are_worth_it(plan):
    rng = np.random.default_rng(12)
    cut = 0
    for T, d, f, gated, dtype in _sizes(rng, 4000):
        bf16 = dtype == "bf16"
        for which in range(6):
            shape, split, M, N, K, segs, outs = plan(which, T, d, f, 1 + gated, bf16)
            assert bf16 or shape in (T128x128, T64x64)
            assert 1 <= split <= 16
            if split > 1:
                cut += 1
                assert split * outs * M * (-(-N // 8) * 8) * 4 <= plan.room
                assert segs * -(-K // (32 if bf16 else 16)) // split >= 4
    assert cut > 1000


def test_the_products_of_the_two_passes(plan):
    """Their sizes, for T tokens of a d x f layer."""
    T, d, f = 40, 64, 203
    want = {UP: (T, f, d), DOWN: (T, d, f), GRAD: (T, f, d), DX: (T, d, f), DUP: (d, f, T), DDOWN: (f, d, T)}
    for which, (M, N, K) in want.items():
        for planes in (1, 2):
            got = plan(which, T, d, f, planes, True)
            assert tuple(got[2:5]) == (M, N, K)
            assert got[5] == (planes if which == DX else 1)
            assert got[6] == (planes if which in (UP, DUP) else 1)


def test_the_scratch_holds_what_is_chosen(plan):
    """Of a product, and of each with one gradient of a gated layer alone: never more than the sized scratch."""
    rng = np.random.default_rng(13)
    sizes = list(_sizes(rng, 6000)) + SIZES + [((1 << 28), 8, 8, True, "bf16"), (1, 8, 8, True, "bf16"), (40, 1 << 20, 200, True, "bf16")]
    for T, d, f, gated, dtype in sizes:
        bf16 = dtype == "bf16"
        for which in range(6):
            room = plan.bytes(which, T, d, f, 1 + gated, bf16)
            assert room <= plan.room and room <= plan.bytes(which, 2 * T, d, f, 1 + gated, bf16)
            for planes in {1 + gated, 1} if which == DUP else {1 + gated}:
                shape, split, M, N, K, segs, outs = plan(which, T, d, f, planes, bf16)
                if split > 1:
                    assert split * outs * M * (-(-N // 8) * 8) * 4 <= room, (which, T, d, f, planes, dtype)
    assert plan.bytes(DUP, 100, 8, 8, 2, True) == 0      # (a reduction that is too short to cut)


def test_small_layers_take_small_scratch():
    import paper_2401_04044_amd as ff
    desc = ff.make_desc(8, 8, "swiglu", "bf16")
    for call in (ff.WS_DENSE_FORWARD, ff.WS_DENSE_BACKWARD):
        assert 0 < ff.workspace_bytes(desc, call, 1) <= 1 << 16
    # (a stack's holds its norm's sums too, of up to 4096 layers)
    assert ff.lib.ffsplit_workspace_bytes(None, ff.WS_GRAD_NORM, 3 * 4096) <= ff.workspace_bytes(desc, ff.WS_DENSE_STACK, 1) <= 1 << 23
    large = ff.make_desc(4096, 11008, "swiglu", "bf16")
    assert ff.workspace_bytes(large, ff.WS_DENSE_FORWARD, 4096) <= 4096 * 11008 * 2 + (64 << 20)
