"""The rules that pick the launches of attention over a cache's rows (csrc/span_plan.h), compiled for the CPU: the GPU tests reach
every kernel, whatever the rules' constants become, and no launch or workspace is outside what the kernels are made for."""
import ctypes as C
import os
import random
import subprocess

import pytest

import test_gpu_span_attn as gpu
from paper_2601_17818_amd import binding as vc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2601_17818_amd", "csrc", "span_plan.h")

WRAPPER = """
#include "%s"
extern "C" void plan(const int64_t* z, int d, int tree, int own, int fits, int* o) {
    const vitcop::SpanPlan p = vitcop::span_plan({z[0], z[1], z[2], z[3], z[4], z[5], z[6], d, tree != 0, own != 0}, fits != 0);
    o[0] = p.wide; o[1] = p.blocks; o[2] = p.row_blocks; o[3] = p.slices;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(WRAPPER % HEADER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    lib = C.CDLL(str(d / "plan.so"))

    def walk(B, Hkv, T, G, start, window, sinks, d, tree, own, fits=True):
        o = (C.c_int * 4)()
        lib.plan((C.c_int64 * 7)(B, Hkv, T, G, start, window, sinks), d, tree, own, fits, o)
        return tuple(o)

    return walk


def test_the_gpu_tests_reach_every_kernel(plan):
    """(d, tree, wide, blocks) and whether slices are merged, few (up to eight) or many."""
    reached = set()

    def note(B, T, start, Hq, Hkv, d, window, sinks, tree, own):
        window = 0 if window >= start + T else window                # (as the call has it)
        sinks = min(sinks, start + T) if window else 0
        wide, blocks, _, slices = plan(B, Hkv, T, Hq // Hkv, start, window, sinks, d, tree, own)
        reached.add((d, tree, wide, blocks))
        reached.add((d, "one slice" if slices == 1 else "few slices" if slices <= 8 else "many slices"))

    for B, T, start, Hq, Hkv, d, window, sinks in gpu.WINDOWS:
        note(B, T, start, Hq, Hkv, d, window, sinks, False, False)
    for B, T, start, Hq, Hkv, d in gpu.TREES:
        note(B, T, start, Hq, Hkv, d, 0, 0, True, False)
    want = {(d, tree, 0, blocks) for d in (64, 128) for tree in (False, True) for blocks in (1, 2)}
    want |= {(d, tree, 1, 1) for d in (64, 128) for tree in (False, True)} | {(128, False, 1, 2)}
    want |= {(d, n) for d in (64, 128) for n in ("one slice", "few slices", "many slices")}
    assert want <= reached, want - reached
    assert reached <= want, reached - want


def test_launches_fit(plan):
    rng = random.Random(1)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))  # noqa: E731
    for _ in range(20000):
        tree = rng.random() < 0.4
        B, Hkv, G = log(1, 65535), log(1, 65535), log(1, 64)
        T = log(1, 64) if tree else log(1, 1 << 20)
        if B * Hkv >= 1 << 23 or B * T * Hkv * G >= 1 << 28:
            continue
        start = rng.choice([0, log(1, (1 << 30) - T)])
        window = rng.choice([0, log(1, 1 << 20)])
        window = 0 if tree or window >= start + T else window
        sinks = min(rng.choice([0, log(1, 1 << 20)]), start + T) if window else 0
        d = rng.choice([64, 128])
        fits = rng.random() < 0.8
        wide, blocks, row_blocks, slices = plan(B, Hkv, T, G, start, window, sinks, d, tree, rng.random() < 0.5, fits)
        rows = T * G
        unit = (128 if wide else 16) * blocks
        assert fits or not wide
        assert wide == int(fits and rows > 32) and blocks in (1, 2) and not (wide and blocks == 2 and (d == 64 or tree))
        assert (row_blocks - 1) * unit < rows <= row_blocks * unit
        assert 1 <= slices <= max(1, 1024 // (B * Hkv * row_blocks))
        assert B * Hkv * row_blocks * slices * 256 < 1 << 32                 # threads of the launch
        assert slices == 1 or B * Hkv * rows * 256 < 1 << 32                 # and of the merge's
        if not wide and rows <= 32:
            assert row_blocks * slices <= 65535


def test_workspaces_hold_the_slices(plan):
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    for B, T, start, Hq, Hkv, d, window, sinks in gpu.WINDOWS:
        window, sinks = (0, 0) if window >= start + T else (window, min(sinks, start + T) if window else 0)
        most = max(plan(B, Hkv, T, Hq // Hkv, start, window, sinks, d, False, own)[3] for own in (False, True))
        want = up(B * T * Hq * most * d * 4) + up(B * T * Hq * most * 8) if most > 1 else 0
        assert vc.lib.vitcop_window_attn_workspace_bytes(B, T, start, Hq, Hkv, d, window, sinks) == want
    for B, T, start, Hq, Hkv, d in gpu.TREES:
        most = max(plan(B, Hkv, T, Hq // Hkv, start, 0, 0, d, True, own)[3] for own in (False, True))
        want = up(B * T * Hq * most * d * 4) + up(B * T * Hq * most * 8) if most > 1 else 0
        assert vc.lib.vitcop_tree_attn_workspace_bytes(B, T, start, Hq, Hkv, d) == want


def test_what_was_measured(plan):
    """The rules take what was quickest, or within a few percent of it, at sizes given in the header."""
    assert plan(1, 32, 1, 1, 300, 0, 0, 128, False, False)[3] == 1
    assert plan(64, 4, 1, 7, 2000, 0, 0, 128, False, False)[3] == 1
    assert plan(1, 4, 1, 7, 16000, 0, 0, 128, False, False)[3] >= 32
    assert plan(1, 4, 317, 7, 16384, 0, 0, 128, False, False) == (1, 2, 9, 7)
    assert plan(1, 32, 640, 1, 0, 0, 0, 128, False, False) == (1, 1, 5, 1)
    assert plan(2, 4, 8192, 7, 0, 2048, 16, 128, False, False) == (1, 2, 224, 1)
    assert plan(8, 4, 64, 7, 4096, 0, 0, 128, True, False) == (1, 1, 4, 2)
    assert plan(64, 4, 1, 7, 16000, 0, 0, 128, False, True)[3] == 2
