"""The rules that pick the launches of the calls on 4-bit caches and matrices (csrc/mx4_plan.h), compiled for the CPU: the GPU
tests reach every kernel, whatever the rules' constants become."""
import ctypes as C
import os
import subprocess

import pytest

import test_gpu_mx4 as gpu
import test_gpu_mx4_attn as gpu_attn
import test_gpu_mx4_project as gpu_project

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2601_17818_amd", "csrc", "mx4_plan.h")

WRAPPER = """
#include "%s"
using namespace vitcop;
extern "C" {
void attn(int B, int N, int Hkv, int d, int* o) {
    const AttnPlan p = attn_plan(B, N, Hkv, d);
    o[0] = p.waves; o[1] = p.splits; o[2] = p.keys_per_split;
}
int products(int heads) { return attn_products(heads); }
void few(int M, int N, int K, int* o) {
    const FewPlan p = few_plan(M, N, K);
    o[0] = p.blocks; o[1] = p.x_loads; o[2] = p.waves; o[3] = p.depth;
}
void project(int M, int N, int K, int* o) {
    const MpPlan p = mp_plan(M, N, K);
    o[0] = p.kind; o[1] = p.slices; o[2] = p.steps_per_slice; o[3] = p.unpack;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(WRAPPER % HEADER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return C.CDLL(str(d / "plan.so"))


def walked(f, n, *sizes):
    o = (C.c_int * n)()
    f(*sizes, o)
    return tuple(o)


def sizes_of(test):
    """The parameters that a GPU test is run with."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize")


ATTENTION = [s for t in (gpu.test_attention, gpu_attn.test_slices_and_wavefronts) for s in sizes_of(t)]
TILES = [s[:3] for t in (gpu.test_projection_on_tiles, gpu.test_projection_of_many_rows,
                                gpu_project.test_projection_on_the_largest_tiles) for s in sizes_of(t)]
FEW = [s for t in (gpu.test_projection, gpu.test_projection_of_long_matrices) for s in sizes_of(t)]


def attention_kernels(plan, B, N, Hq, Hkv, d):
    """(head dimension, wavefronts, sliced, products) of the passes of a call."""
    waves, splits, _ = walked(plan.attn, 3, B, N, Hkv, d)
    return {(d, waves, splits > 1, plan.products(min(16, Hq // Hkv - g0))) for g0 in range(0, Hq // Hkv, 16)}


def test_gpu_tests_reach_every_attention_kernel(plan):
    reached = set().union(*(attention_kernels(plan, *s) for s in ATTENTION))
    missing = {(d, w, cut, n) for d in (64, 128) for w, cut in ((2, False), (4, False), (8, False), (4, True), (8, True))
               for n in (1, 2, 3)} - reached
    assert not missing, sorted(missing)


def test_slices_of_the_keys(plan):
    """None of them without a key, whole tiles of keys to a wavefront, and no more workgroups than are of use."""
    for d in (64, 128):
        for B, Hkv in ((1, 1), (1, 32), (3, 5), (7, 4), (31, 1), (8, 16), (33, 4), (64, 4), (20, 16), (65, 8), (700, 3), (3000, 1)):
            for N in (0, 1, 31, 32, 33, 160, 161, 400, 800, 801, 1500, 1501, 8193, 40000, 65536, 1 << 20, (1 << 31) // d - 1):
                waves, splits, keys = walked(plan.attn, 3, B, N, Hkv, d)
                assert waves in (2, 4, 8) and keys % (32 * waves) == 0 or keys == 2 ** 31 - 1
                assert splits >= 1 and splits * keys >= N and (splits == 1 or (splits - 1) * keys < N)
                assert splits == 1 or B * Hkv * splits <= 2048


def test_gpu_tests_reach_every_kernel_of_few_rows(plan):
    reached = {walked(plan.few, 4, *s) for s in FEW + TILES if walked(plan.project, 4, *s)[0] < 0}
    taken = {walked(plan.few, 4, M, N, K) for M in (*range(1, 18), 64) for N in (16, 4096, 4112, 8192, 8208, 12288, 12304, 16400, 28672)
             for K in (32, 1024, 1056, 2048, 2080, 4096, 16384, 32768, 32800, 65536) if N * K < 1 << 31}
    assert taken == reached | {walked(plan.few, 4, 9, 12320, 32800)} and len(taken) == 13


def test_gpu_tests_reach_every_tile(plan):
    """Each kind, in one slice and in several, K a whole number of steps and not."""
    reached = {(p[0], p[1] > 1, s[2] % 128 == 0) for s in TILES for p in [walked(plan.project, 4, *s)] if not p[3]}
    missing = {(kind, cut, whole) for kind in range(8) for cut in (False, True) for whole in (False, True)} - reached
    assert not missing, sorted(missing)
    assert any(walked(plan.project, 4, *s)[3] for s in TILES)


def test_slices_of_k(plan):
    """None empty, each of four steps at least."""
    for M in (17, 33, 64, 150, 317, 700, 1100):
        for N, K in ((16, 512), (512, 3584), (4096, 4096), (4096, 11008), (3584, 14336), (272, 4128), (8192, 65536)):
            kind, slices, steps, _ = walked(plan.project, 4, M, N, K)
            if kind >= 0:
                total = (K + 127) // 128
                assert slices * steps >= total and (slices - 1) * steps < total and (slices == 1 or steps >= 4)


@pytest.mark.parametrize("pairs,N,d,sliced", [
    # us in one slice and in slices: 7.6, 7.9; 8.8, 7.5; 8.2, 9.2; 9.1, 9.3; 10.1, 9.4; 10.3, 10.6; 11.6, 10.9
    (64, 650, 128, False), (16, 1000, 128, True), (96, 801, 128, False), (96, 1000, 128, False), (96, 1200, 128, True),
    (128, 1200, 128, False), (128, 1500, 128, True),
    # 6.2, 6.8; 7.6, 7.0; 7.1, 7.4; 8.7, 8.0; 8.0, 8.9; 10.5, 9.9
    (16, 801, 64, False), (16, 1200, 64, True), (64, 1000, 64, False), (64, 1500, 64, True), (128, 1200, 64, False),
    (128, 2000, 64, True)])
def test_few_keys_are_not_sliced(plan, pairs, N, d, sliced):
    for B, Hkv in ((pairs, 1), (pairs // 8, 8)):
        assert (walked(plan.attn, 3, B, N, Hkv, d)[1] > 1) == sliced


@pytest.mark.parametrize("M,N,K,blocks", [
    # us with one and with two blocks of 16 rows of the matrix to a workgroup: 7.2, 7.9; 8.4, 8.2; 10.7, 11.2; 13.2, 14.0;
    # 24.8, 22.6; 15.6, 14.3; 9.2, 8.7
    (2, 12288, 4096, 1), (2, 14336, 4096, 2), (2, 20480, 4096, 1), (2, 28672, 4096, 1), (2, 14336, 14336, 2), (2, 12800, 8192, 2),
    (2, 57344, 1024, 2),
    # one row: 23.5, 22.5; 14.7, 14.2; 6.0, 5.7; 10.5, 11.1; 7.0, 7.6
    (1, 14336, 14336, 2), (1, 12800, 8192, 2), (1, 16384, 2048, 2), (1, 20480, 4096, 1), (1, 11008, 4096, 1),
    # up to 512 blocks: 10.1, 9.6; 6.1, 5.7
    (4, 8192, 8192, 2), (4, 6144, 4096, 2)])
def test_blocks_of_few_rows(plan, M, N, K, blocks):
    assert walked(plan.few, 4, M, N, K)[0] == blocks
