"""GPU parity: rows of a KV cache in 4 bits, written and read at a wavefront's own boundaries, and refusals that write nothing."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import mx4_oracle as X
from gpu_util import dev, host_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vc():
    from paper_2601_17818_amd import binding
    return binding


def filled(vc, B, capacity, Hkv, d, byte=0x5A):
    cache = vc.CacheMx4.empty(B, capacity, Hkv, d)
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.fill_(byte)
    return cache


def tensors(cache):
    return [t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


# a wavefront takes 8 tokens of heads of 128, 16 of heads of 64, in two loads each
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [3, 4, 5, 7, 8, 9, 15, 16, 17, 24, 25, 33])
def test_rows_around_a_wavefronts_own(vc, T, d):
    B, Hkv, capacity, start = 2, 3, 40, 4
    rows = [I.normal_bf16(T + d, i, (B, T, Hkv, d)) for i in range(2)]
    counts = [T, max(T - 1, 0)]
    for n in (None, counts):
        cache = filled(vc, B, capacity, Hkv, d)
        want = tensors(cache)
        for side in range(2):
            codes, scales = X.quantize(rows[side])
            for b in range(B):
                m = T if n is None else n[b]
                want[2 * side][b, :, start:start + m] = codes[b, :m].transpose(1, 0, 2)
                want[2 * side + 1][b, :, start:start + m] = scales[b, :m].transpose(1, 0, 2)
        vc.vitcop_cache_mx4_write(cache, dev(rows[0]), dev(rows[1]), start,
                                  n_samples=None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda"))
        assert all(np.array_equal(a, b) for a, b in zip(tensors(cache), want))
        for side, x in enumerate(vc.vitcop_cache_mx4_read(cache, T, start)):
            held = X.values(want[2 * side], want[2 * side + 1])[:, :, start:start + T].transpose(0, 2, 1, 3)
            assert np.array_equal(host_f64(x), held)


def test_a_refused_write_writes_nothing(vc):
    # K is in order and V is not, each with strides of its own: neither side may change
    B, T, Hkv, d = 2, 5, 2, 64
    k = dev(I.normal_bf16(1, 0, (B, T, Hkv, d)))
    wide = torch.zeros((B, T, Hkv * d + 12), dtype=torch.bfloat16, device="cuda")
    apart = torch.zeros(B * (T * Hkv * d + 4), dtype=torch.bfloat16, device="cuda")
    shifted = torch.zeros(B * T * (Hkv * d + 8) + 8, dtype=torch.bfloat16, device="cuda")
    bad = [wide[:, :, :Hkv * d].unflatten(-1, (Hkv, d)),                                          # rows 140 elements apart
           apart.as_strided((B, T, Hkv, d), (T * Hkv * d + 4, Hkv * d, d, 1)),                    # samples 644 apart
           shifted.as_strided((B, T, Hkv, d), (T * (Hkv * d + 8), Hkv * d + 8, d, 1), 4)]         # 8 bytes off
    cache = filled(vc, B, 16, Hkv, d)
    before = tensors(cache)
    for x in bad:
        for pair in ((k, x), (x, k)):
            with pytest.raises((ValueError, vc.VitcopError)):
                vc.vitcop_cache_mx4_write(cache, *pair)
            assert all(np.array_equal(a, b) for a, b in zip(tensors(cache), before))
    one = torch.zeros((1, T, Hkv, d), dtype=torch.bfloat16, device="cuda")
    vc.vitcop_cache_mx4_write(cache, k, one.expand(B, T, Hkv, d))                                 # two layouts, both in order
    assert not np.array_equal(tensors(cache)[0], before[0]) and not np.array_equal(tensors(cache)[2], before[2])


def test_sizes_past_32_bits_are_refused(vc):
    # the C calls take 32-bit sizes: 2^32 + n must not be taken for n
    past = 1 << 32
    k = dev(I.normal_bf16(2, 0, (1, 1, 2, 64)))
    cache = filled(vc, 1, 16, 2, 64)
    before = tensors(cache)
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    long_row = torch.empty((1, past + 32), dtype=torch.bfloat16, device="cuda")
    long_codes = torch.empty((1, past // 2 + 16), dtype=torch.uint8, device="cuda")
    long_scales = torch.empty((1, past // 32 + 1), dtype=torch.uint8, device="cuda")
    for bad in (lambda: vc.vitcop_cache_mx4_write(cache, k, None, past), lambda: vc.vitcop_cache_mx4_write(cache, k, k, 2 - past),
                lambda: vc.vitcop_cache_mx4_write(cache, k.expand(1, past + 1, 2, 64), None),
                lambda: vc.vitcop_cache_mx4_read(cache, 1, past), lambda: vc.vitcop_decode_attn_mx4(q, cache, past + 3),
                lambda: vc.vitcop_mx4_quantize(long_row), lambda: vc.vitcop_mx4_dequantize(long_codes, long_scales),
                lambda: vc.vitcop_project_mx4(long_row, long_codes, long_scales)):
        with pytest.raises((ValueError, vc.VitcopError)):
            bad()
    assert all(np.array_equal(a, b) for a, b in zip(tensors(cache), before))


def test_nothing_to_write_is_refused(vc):
    with pytest.raises(ValueError):
        vc.vitcop_cache_mx4_write(filled(vc, 1, 16, 2, 64), None, None)


def test_a_caches_tensors_stay_its_own(vc):
    # the descriptor holds their addresses: another tensor in the place of one would not be seen
    cache = filled(vc, 1, 16, 2, 64)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales", "B", "Hkv", "capacity", "d"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name))
