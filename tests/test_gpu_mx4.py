"""GPU parity: rows, KV caches and weights in 4 bits and the decoding over them, against the float64 oracle.

Bounds.  What is held in 4 bits is compared for equality.  A bf16 output is off by half a step, 2^-8 of itself, and by what
the fp32 sums before it carry: n products summed in fp32 are off by at most (n + 2) 2^-24 of the sum of their magnitudes.
"""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import decoder_oracle as Dc
from oracle import mx4_oracle as X
from oracle import vitcop_oracle as O
from gpu_util import dev, host_bits, host_f64

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def vc():
    from paper_2601_17818_amd import binding
    return binding


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def same_values(got: torch.Tensor, want: np.ndarray, what=""):
    got = host_f64(got)
    assert np.array_equal(got, want, equal_nan=True), what
    assert np.array_equal(np.signbit(got[got == 0]), np.signbit(want[want == 0])), what + " (signs of zeros)"


# ------------------------------------------------------------------------------------------------- rows


# rows of one group, odd numbers of groups, a row that ends inside a thread block's share, one below and above it
@pytest.mark.parametrize("M,K", [(1, 32), (3, 96), (7, 1056), (1, 8192), (5, 8224), (130, 4096), (2816, 1024)])
def test_rows_there_and_back(vc, M, K):
    x = I.normal_bf16(100 + M, 0, (M, K))
    x[0, :4] = [0, 0x8000, 0x0001, 0x8040]                                # zeros of both signs, denormal values
    codes, scales = vc.vitcop_mx4_quantize(dev(x))
    want_c, want_s = X.quantize(x)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    same_values(vc.vitcop_mx4_dequantize(codes, scales), X.values(want_c, want_s))


def test_every_bf16_next_to_every_size_of_a_group(vc):
    # all 65536 bit patterns, each in groups whose largest value gives exponents from the lowest to the highest
    every = np.arange(65536, dtype=np.uint16)
    tops = [0x0000, 0x0100, 0x0160, 0x0161, 0x1234, 0x3F80, 0x40E0, 0x40E1, 0x6000, 0x7E60, 0x7E61, 0x7F7F]
    x = np.zeros((len(tops), 65536 // 16, 32), np.uint16)
    for t, top in enumerate(tops):
        x[t, :, :16] = every.reshape(-1, 16)
        x[t, :, 16] = top
    x = x.reshape(len(tops), -1)
    codes, scales = vc.vitcop_mx4_quantize(dev(x))
    want_c, want_s = X.quantize(x)
    assert np.array_equal(scales.cpu().numpy(), want_s) and np.array_equal(codes.cpu().numpy(), want_c)
    same_values(vc.vitcop_mx4_dequantize(codes, scales), X.values(want_c, want_s))


def test_every_code_and_exponent_reads_back(vc):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))             # [256 exponents, 512 values]
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    keep = [s for s in range(256) if s not in (253, 254)]                 # (may stand for infinities)
    got = vc.vitcop_mx4_dequantize(u8(codes), u8(scales))
    same_values(got[keep], X.values(codes, scales)[keep])


def test_strided_rows(vc):
    wide = I.normal_bf16(7, 0, (9, 256))
    x = dev(wide)[:, 64:192]                                              # rows 256 apart
    codes, scales = vc.vitcop_mx4_quantize(x)
    want = X.quantize(wide[:, 64:192])
    assert np.array_equal(codes.cpu().numpy(), want[0]) and np.array_equal(scales.cpu().numpy(), want[1])
    out = torch.full((9, 256), 3.0, dtype=torch.bfloat16, device="cuda")
    vc.vitcop_mx4_dequantize(codes, scales, out=out[:, 64:192])
    same_values(out[:, 64:192].contiguous(), X.values(*want))
    assert (out[:, :64] == 3).all() and (out[:, 192:] == 3).all()


# ------------------------------------------------------------------------------------------------ cache


def filled(vc, seed, B, capacity, Hkv, d):
    """A cache of other contents, and those as float64 [B,Hkv,capacity,d] (K, V)."""
    rng = np.random.default_rng(seed)
    raw = []
    for _ in range(2):
        raw += [rng.integers(0, 256, (B, Hkv, capacity, d // 2)).astype(np.uint8),
                rng.integers(100, 150, (B, Hkv, capacity, d // 32)).astype(np.uint8)]
    return vc.CacheMx4(*[u8(a) for a in raw]), [X.values(raw[0], raw[1]), X.values(raw[2], raw[3])]


def contents(cache):
    return [X.values(c.cpu().numpy(), s.cpu().numpy())
            for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))]


# one token, a wavefront's tokens (32 of d = 128, 64 of d = 64), one fewer and more, several; odd head counts
@pytest.mark.parametrize("B,T,Hkv,d,capacity,start", [
    (1, 1, 1, 64, 1, 0), (3, 1, 5, 128, 9, 8), (2, 31, 3, 128, 40, 9), (2, 32, 4, 128, 33, 0), (1, 33, 7, 128, 64, 31),
    (2, 63, 2, 64, 70, 3), (1, 65, 3, 64, 65, 0), (2, 300, 4, 128, 333, 11), (5, 7, 32, 128, 16, 2)])
def test_cache_rows_and_nothing_else(vc, B, T, Hkv, d, capacity, start):
    cache, want = filled(vc, T + d, B, capacity, Hkv, d)
    t = [I.normal_bf16(200 + T, i, (B, T, Hkv, d)) for i in range(2)]
    vc.vitcop_cache_mx4_write(cache, dev(t[0]), dev(t[1]), start)
    for side in range(2):
        want[side][:, :, start:start + T] = X.round_trip(t[side]).transpose(0, 2, 1, 3)
        assert np.array_equal(contents(cache)[side], want[side])
    back = vc.vitcop_cache_mx4_read(cache, T, start)
    for side in range(2):
        same_values(back[side], X.round_trip(t[side]))
    whole = vc.vitcop_cache_mx4_read(cache, capacity)
    for side in range(2):
        assert np.array_equal(host_f64(whole[side]), want[side].transpose(0, 2, 1, 3))


def test_rows_at_every_samples_own_place(vc):
    # counts from none to more than there are, starts before, inside and past the cache: outside rows are skipped,
    # and read as zeros
    B, T, Hkv, d, capacity = 8, 40, 3, 128, 50
    start = [0, 10, 30, 49, -7, 50, -100, 2147483647]
    count = [40, 0, 40, 40, 40, 3, 40, 41]
    cache, want = filled(vc, 1, B, capacity, Hkv, d)
    before = [w.copy() for w in want]
    t = [I.normal_bf16(300, i, (B, T, Hkv, d)) for i in range(2)]
    vc.vitcop_cache_mx4_write(cache, dev(t[0]), dev(t[1]), start_samples=i32(start), n_samples=i32(count))
    back = vc.vitcop_cache_mx4_read(cache, T, start_samples=i32(start))
    for side in range(2):
        held = X.round_trip(t[side])
        read = np.zeros((B, T, Hkv, d))
        for b in range(B):
            for r in range(T):
                if 0 <= start[b] + r < capacity:
                    if r < count[b]:
                        want[side][b, :, start[b] + r] = held[b, r]
                    read[b, r] = want[side][b, :, start[b] + r]
        assert np.array_equal(contents(cache)[side], want[side])
        assert np.array_equal(host_f64(back[side]), read)
    n = i32([-5] * B)
    vc.vitcop_cache_mx4_write(cache, dev(t[0]), dev(t[1]), 0, n_samples=n)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want)) and not np.array_equal(before[0], want[0])


def test_strided_and_single_sides(vc):
    # K and V inside fused rows, a batch dimension inside the token's, one side alone, K and V of different strides
    B, T, Hkv, d = 3, 20, 4, 64
    rows = I.normal_bf16(400, 0, (B, T, 3, Hkv, d))
    q, k, v = (dev(rows)[:, :, i] for i in range(3))
    cache, want = filled(vc, 2, B, 32, Hkv, d)
    vc.vitcop_cache_mx4_write(cache, k, None, 5)
    want[0][:, :, 5:25] = X.round_trip(rows[:, :, 1]).transpose(0, 2, 1, 3)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want))
    vc.vitcop_cache_mx4_write(cache, None, v, 5)
    want[1][:, :, 5:25] = X.round_trip(rows[:, :, 2]).transpose(0, 2, 1, 3)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want))
    vc.vitcop_cache_mx4_write(cache, v, k, 12)                            # both strided alike
    want[0][:, :, 12:32] = X.round_trip(rows[:, :, 2]).transpose(0, 2, 1, 3)
    want[1][:, :, 12:32] = X.round_trip(rows[:, :, 1]).transpose(0, 2, 1, 3)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want))
    token_major = dev(rows[:, :, 0].transpose(1, 0, 2, 3)).transpose(0, 1)           # [B,T,..] over [T,B,..]
    vc.vitcop_cache_mx4_write(cache, token_major, k, 0)                   # two layouts
    want[0][:, :, :20] = X.round_trip(rows[:, :, 0]).transpose(0, 2, 1, 3)
    want[1][:, :, :20] = X.round_trip(rows[:, :, 1]).transpose(0, 2, 1, 3)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want))
    vc.vitcop_cache_mx4_write(cache, k[:1, :1].expand(B, T, Hkv, d), None, 1)        # one token for all
    want[0][:, :, 1:21] = X.round_trip(rows[:1, :1, 1]).transpose(0, 2, 1, 3)
    assert all(np.array_equal(a, b) for a, b in zip(contents(cache), want))
    only = torch.empty((B, 6, Hkv, d), dtype=torch.bfloat16, device="cuda")
    assert vc.vitcop_cache_mx4_read(cache, 6, 2, out=(None, only))[0] is None
    assert np.array_equal(host_f64(only), want[1][:, :, 2:8].transpose(0, 2, 1, 3))


# -------------------------------------------------------------------------------------------- attention


def attn_check(vc, cache, kv, q, N, lens=None, scale=0.0, what=""):
    """kv: float64 [B,Hkv,capacity,d]; returns (out, lse) as float64 after comparing with the oracle."""
    o, lse = vc.vitcop_decode_attn_mx4(dev(q), cache, N, None if lens is None else i32(lens), scale)
    few = 4 if q.shape[0] > 4 and lens is None else q.shape[0]             # (attn_case: the others repeat them)
    of = np.arange(q.shape[0]) % few
    ref, ref_lse, spread, size = (x[of] for x in X.decode_attention(q[:few], kv[0][:few, :, :N], kv[1][:few, :, :N], lens, scale))
    got, got_lse = host_f64(o), lse.cpu().numpy().astype(np.float64)
    d = q.shape[-1]
    # a score is off by (d + 4) 2^-24 of its products' magnitudes, a probability by that, by 2^-16 of itself as the sum of two
    # bf16 and by the exponential's last bits; numerator and denominator are sums over N
    p_off = (d + 4) * EPS * size + 2.0 ** -16 + 2.0 ** -20 + N * EPS
    assert np.array_equal(np.isneginf(got_lse), np.isneginf(ref_lse)), what
    live = ~np.isneginf(ref_lse)
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * p_off[..., None] * spread)[live].all(), what
    assert not got[~live].any(), what
    assert (np.abs(got_lse[live] - ref_lse[live]) <= p_off[live] + 2.0 ** -22 * (1 + np.abs(ref_lse[live]))).all(), what
    return got, got_lse


def attn_case(vc, seed, B, N, Hq, Hkv, d, capacity=None, std=1.0):
    """A cache of N rows a sample (the others hold NaN), what they stand for, and queries; of more than four samples, four
    different ones dealt out (and of more than sixteen the values of the first four alone)."""
    t = I.qkv_tensors(seed, min(B, 4), N, Hq, Hkv, d, std=std)
    of = np.arange(B) % 4 if B > 4 else np.arange(B)
    cache = vc.CacheMx4.empty(B, capacity or N, Hkv, d)
    for held in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        held.fill_(255)
    vc.vitcop_cache_mx4_write(cache, dev(t["k"])[of], dev(t["v"])[of], 0)
    kv = [X.round_trip(t[n]).transpose(0, 2, 1, 3) for n in ("k", "v")]
    return cache, kv if B > 16 else [x[of] for x in kv], np.ascontiguousarray(t["q"][of, -1])


# one key, a tile of 16 and 32 keys and a workgroup's 128, one fewer and one more, several slices, one; one query head to a KV
# head and 2, 3, 7, 16, 17 (a second pass), 34; one KV head and many
@pytest.mark.parametrize("B,N,Hq,Hkv,d", [
    (1, 1, 1, 1, 64), (1, 1, 2, 2, 128), (2, 15, 4, 4, 64), (2, 16, 4, 2, 128), (2, 17, 4, 2, 64), (2, 31, 4, 2, 128),
    (2, 32, 6, 2, 128), (1, 33, 7, 1, 64), (3, 127, 16, 1, 128), (1, 128, 32, 32, 128), (2, 129, 17, 1, 64), (3, 257, 34, 2, 128),
    (1, 640, 32, 32, 128), (2, 1000, 20, 2, 128), (1, 6400, 28, 4, 128), (70, 160, 28, 4, 128), (40, 70, 32, 32, 64),
    (12, 300, 32, 32, 128), (400, 33, 4, 2, 64), (52, 1100, 15, 15, 64), (9, 3500, 16, 16, 128), (12, 13001, 4, 4, 64),
    (40, 1610, 16, 16, 64), (20, 7001, 28, 14, 64), (96, 900, 28, 14, 128),
    (1, 801, 64, 64, 128), (1, 800, 64, 64, 64), (2, 9001, 4, 2, 128), (1, 20000, 2, 1, 64),
    (1, 4097, 3, 3, 64)])
def test_attention(vc, B, N, Hq, Hkv, d):
    attn_check(vc, *attn_case(vc, 500 + N + Hq, B, N, Hq, Hkv, d), N)


# lengths from none to more than N (clamped), with slices that no key of a sample falls into; the cache's other rows are NaN
@pytest.mark.parametrize("N,Hq,Hkv,d", [(60, 4, 4, 64), (300, 8, 2, 128), (2000, 6, 1, 64), (513, 4, 4, 128)])
def test_attention_of_different_lengths(vc, N, Hq, Hkv, d):
    lens = [N, 0, 1, 31, 32, 33, N // 2, N - 1, 129]
    cache, kv, q = attn_case(vc, 600 + N, len(lens), N, Hq, Hkv, d, capacity=N + 5)
    lens = [min(n, N) for n in lens]
    for b, n in enumerate(lens):
        for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
            t[b, :, n:] = 255
    attn_check(vc, cache, kv, q, N, lens)
    first = vc.CacheMx4(*[t[:1].contiguous() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)])
    assert torch.equal(vc.vitcop_decode_attn_mx4(dev(q[:1]), first, N, i32([N + 77]))[0],
                       vc.vitcop_decode_attn_mx4(dev(q[:1]), first, N)[0])
    none, none_lse = vc.vitcop_decode_attn_mx4(dev(q), cache, N, i32([-3] * len(lens)))
    assert not none.any() and torch.isneginf(none_lse).all()
    zero, zero_lse = vc.vitcop_decode_attn_mx4(dev(q), cache, 0)
    assert not zero.any() and torch.isneginf(zero_lse).all()


def test_attention_scale_and_large_scores(vc):
    # scores from -300 to 300: the reference of the softmax moves often and by much
    cache, kv, q = attn_case(vc, 700, 2, 700, 8, 2, 128, std=4.0)
    attn_check(vc, cache, kv, q, 700)
    attn_check(vc, cache, kv, q, 700, scale=0.3)
    # ascending scores, so that it moves with every tile
    k = O.bf16_to_f64(np.tile(q[:, :1, None], (1, 2, 700, 1))) * (np.arange(700) / 350.0)[None, None, :, None]
    bits = O.f64_to_bf16_bits(k.transpose(0, 2, 1, 3))
    vc.vitcop_cache_mx4_write(cache, dev(bits), None)
    kv[0][:] = X.round_trip(bits).transpose(0, 2, 1, 3)
    attn_check(vc, cache, kv, q, 700)


def test_attention_is_that_of_the_values_read_back(vc):
    # against the framework's attention over the same values as bf16, which rounds its probabilities no further
    cache, kv, q = attn_case(vc, 800, 3, 500, 14, 2, 128)
    k, v = vc.vitcop_cache_mx4_read(cache, 500)
    a, la = vc.vitcop_decode_attn_mx4(dev(q), cache, 500)
    b, lb = vc.vitcop_decode_attn(dev(q), k, v)
    assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-4).all() and (la - lb).abs().max() < 1e-5


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 2, 128)])
def test_a_group_that_is_not_a_number(vc, Hq, Hkv, d):
    # of V: its channels of the KV head's query heads; of K: all channels of them; of a row past the end: nothing
    B, N, G = 2, 200, Hq // Hkv
    cache, kv, q = attn_case(vc, 900, B, N, Hq, Hkv, d, capacity=201)
    plain, _ = attn_check(vc, cache, kv, q, N)
    cache.v_scales[1, 1, 77, 1] = 255
    got = host_f64(vc.vitcop_decode_attn_mx4(dev(q), cache, N)[0])
    want = plain.copy()
    want[1, G:2 * G, 32:64] = np.nan
    assert np.array_equal(got, want, equal_nan=True)
    cache.k_scales[0, 0, 199, 0] = 255
    got = host_f64(vc.vitcop_decode_attn_mx4(dev(q), cache, N)[0])
    want[0, :G] = np.nan
    assert np.array_equal(got, want, equal_nan=True)


def test_a_cache_whose_offsets_pass_32_bits(vc):
    # 2^31 bytes and more of codes before the last sample's rows
    B, Hkv, d, capacity = 3, 64, 128, 300_000
    cache = vc.CacheMx4.empty(B, capacity, Hkv, d)
    assert cache.k_codes.numel() // B * (B - 1) > 1 << 31
    t = I.qkv_tensors(950, 1, 90, Hkv, Hkv, d)
    q = np.repeat(t["q"][:, -1], B, 0)
    n = [0, 0, 90]
    start = i32([0, 0, capacity - 90])
    k, v = (dev(np.repeat(t[x], B, 0)) for x in ("k", "v"))
    vc.vitcop_cache_mx4_write(cache, k, v, start_samples=start, n_samples=i32(n))
    back = vc.vitcop_cache_mx4_read(cache, 90, start_samples=start)
    for side, x in enumerate(("k", "v")):
        same_values(back[side][2:], X.round_trip(t[x]))
    vc.vitcop_cache_mx4_write(cache, k, v, n_samples=i32(n))
    o, lse = vc.vitcop_decode_attn_mx4(dev(q), cache, capacity, i32(n))
    one, kv, q1 = attn_case(vc, 950, 1, 90, Hkv, Hkv, d)
    ref, ref_lse, _, _ = X.decode_attention(q1, kv[0], kv[1])
    assert (np.abs(host_f64(o)[2] - ref[0]) <= 2.0 ** -8 * np.abs(ref[0]) + 1e-3).all()
    assert not o[:2].any() and torch.isneginf(lse[:2]).all()


# ------------------------------------------------------------------------------------------- projection


def project_check(vc, M, N, K, residual, seed=0, x=None, one_slice=False):
    w = I.normal_bf16(1000 + seed + N, 0, (N, K), std=1.28 / np.sqrt(K))
    x = I.normal_bf16(1001 + seed + M, 1, (M, K)) if x is None else x
    r = I.normal_bf16(1002 + seed + M, 2, (M, N)) if residual else None
    codes, scales = vc.vitcop_mx4_quantize(dev(w))
    y = vc.vitcop_project_mx4(dev(x), codes, scales, residual=None if r is None else dev(r))
    wv, xv = X.values(codes.cpu().numpy(), scales.cpu().numpy()), O.bf16_to_f64(x)
    ref, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    if r is not None:
        ref, size = ref + O.bf16_to_f64(r), size + np.abs(O.bf16_to_f64(r))
    bound = 2.0 ** -8 * np.abs(ref) + (K + 4) * EPS * size
    assert (np.abs(host_f64(y) - ref) <= bound).all(), (M, N, K)
    if one_slice:                # without scratch: the same sums in another order where k would be cut
        one = vc.vitcop_project_mx4(dev(x), codes, scales, residual=None if r is None else dev(r),
                                    ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
        assert (np.abs(host_f64(one) - ref) <= bound).all(), (M, N, K)
        assert vc.lib.vitcop_project_mx4_workspace_bytes(M, N, K) > 0 or torch.equal(one, y)
    return y


# columns: one group, less and more than a step of 128, not a multiple of it, more than the wavefronts' first turn; rows of the
# matrix: 16, 32, not a multiple of 32; rows of x on both sides of every block of 16 and 64, and many
@pytest.mark.parametrize("M,N,K", [
    (1, 16, 32), (1, 48, 96), (2, 32, 128), (3, 16, 160), (1, 4096, 4096), (4, 272, 1056), (5, 80, 2048), (15, 64, 512),
    (16, 48, 1024), (17, 48, 1024), (32, 112, 544), (33, 80, 672), (63, 48, 256), (64, 1024, 2816), (65, 96, 320), (130, 48, 1152),
    (317, 256, 1024), (7, 3584, 14336), (1, 11008, 4096), (1024, 64, 64)])
def test_projection(vc, M, N, K):
    project_check(vc, M, N, K, residual=(M + N // 16) % 2 == 0)


# sixteen rows of x at a time over a matrix of more 16-row blocks than 256, 512 and 768, of which workgroups take one, two,
# three or four (a last one that is not full), with four and eight wavefronts; and fewer than 512 columns for many rows of x
@pytest.mark.parametrize("M,N,K", [
    (2, 1040, 1056), (3, 4112, 2080), (4, 4112, 96), (2, 12304, 96), (1, 8224, 160), (4, 12320, 544), (7, 2064, 2080),
    (6, 4112, 96), (8, 8240, 288), (8, 12320, 96), (16, 12304, 160), (16, 4112, 160), (13, 8272, 224), (40, 8272, 96),
    (31, 4144, 480), (700, 4096, 256)])
def test_projection_of_long_matrices(vc, M, N, K):
    project_check(vc, M, N, K, residual=M % 2 == 0, seed=8)


def test_projection_of_wide_and_long_matrices(vc):
    # too many columns for the exponents of 64 rows: each row of the matrix as in a short one, whose sums run in the same order
    M, N, K = 9, 12320, 32800
    gen = torch.Generator("cuda").manual_seed(5)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scales = torch.randint(118, 124, (N, K // 32), dtype=torch.uint8, device="cuda", generator=gen)
    x = dev(I.normal_bf16(1150, 0, (M, K)))
    y = vc.vitcop_project_mx4(x, codes, scales)
    for n in (0, 4096, N - 32):
        assert torch.equal(y[:, n:n + 32], vc.vitcop_project_mx4(x, codes[n:n + 32], scales[n:n + 32]))


# tiles of 32 rows of x to 160 by 128 and by 256 rows of the matrix, in one slice of k and in several, with K a whole number of
# steps of 128 and not (its rows of exponents then start at every byte of a word), N no whole number of tiles
@pytest.mark.parametrize("M,N,K", [
    (317, 2272, 608), (316, 640, 4448), (306, 464, 6784), (323, 608, 5632), (20, 8208, 4352), (294, 3392, 640), (313, 448, 6976),
    (320, 672, 4864), (328, 6288, 544), (323, 1472, 3168), (284, 1040, 6656), (329, 1424, 6208), (322, 1520, 6144),
    (297, 2256, 4448), (318, 2304, 4480), (298, 8224, 512), (259, 3696, 544), (328, 5440, 512), (524, 6736, 544), (388, 8240, 512),
    (210, 1488, 512), (399, 6624, 544), (99, 5584, 3840), (109, 5424, 4512), (101, 5408, 4608), (130, 3088, 7296),
    (99, 4160, 5056), (132, 2848, 7008), (129, 6720, 5760), (690, 8208, 576), (674, 8240, 640), (131, 8272, 4320),
    (65, 6640, 5728), (489, 8208, 512), (67, 6560, 5760), (516, 8272, 544), (110, 8304, 4480), (100, 8208, 4416),
    (129, 6608, 6784), (141, 8240, 5152)])
def test_projection_on_tiles(vc, M, N, K):
    project_check(vc, M, N, K, residual=M % 2 == 0, seed=7, one_slice=True)


# many rows over a short matrix: tiles in several rounds; over a larger one: the matrix to bf16 first, and the same
# with no scratch, tiles in several rounds
@pytest.mark.parametrize("M,N,K,unpacked", [(8192, 1024, 1024, False), (5003, 2064, 1056, True), (5003, 2064, 2080, True)])
def test_projection_of_many_rows(vc, M, N, K, unpacked):
    assert (vc.lib.vitcop_project_mx4_workspace_bytes(M, N, K) >= 2 * N * K) == unpacked
    project_check(vc, M, N, K, residual=M % 2 == 1, seed=9, one_slice=True)


def test_projection_of_many_rows_strided_and_in_place(vc):
    M, N, K = 2600, 4112, 2080
    assert vc.lib.vitcop_project_mx4_workspace_bytes(M, N, K) >= 2 * N * K
    codes, scales = vc.vitcop_mx4_quantize(dev(I.normal_bf16(1110, 0, (N, K))))
    x = torch.full((M, K + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = torch.full((M, N + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    xb, rb = I.normal_bf16(1111, 0, (M, K)), I.normal_bf16(1112, 0, (M, N))
    x[:, 32:32 + K], y[:, 8:8 + N] = dev(xb), dev(rb)
    vc.vitcop_project_mx4(x[:, 32:32 + K], codes, scales, residual=y[:, 8:8 + N], out=y[:, 8:8 + N])
    want = vc.vitcop_project_mx4(dev(xb), codes, scales, residual=dev(rb))
    assert torch.equal(y[:, 8:8 + N], want) and (y[:, :8] == 5).all() and (y[:, 8 + N:] == 5).all()


def test_projection_strided(vc):
    # rows of x, y and the residual inside wider ones; what lies between them stays, and is not read: NaN
    M, N, K = 21, 48, 96
    w = I.normal_bf16(1100, 0, (N, K))
    codes, scales = vc.vitcop_mx4_quantize(dev(w))
    x = torch.full((M, 160), float("nan"), dtype=torch.bfloat16, device="cuda")
    r = torch.full((M, 80), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = torch.full((M, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    xb, rb = I.normal_bf16(1101, 0, (M, K)), I.normal_bf16(1102, 0, (M, N))
    x[:, 32:32 + K], r[:, 16:16 + N] = dev(xb), dev(rb)
    vc.vitcop_project_mx4(x[:, 32:32 + K], codes, scales, residual=r[:, 16:16 + N], out=y[:, 8:8 + N])
    want = vc.vitcop_project_mx4(dev(xb), codes, scales, residual=dev(rb))
    assert torch.equal(y[:, 8:8 + N], want) and (y[:, :8] == 5).all() and (y[:, 8 + N:] == 5).all()


def test_projection_in_place_of_the_residual_and_not_a_number(vc):
    M, N, K = 9, 64, 256
    w = I.normal_bf16(1200, 0, (N, K))
    codes, scales = vc.vitcop_mx4_quantize(dev(w))
    x, r = I.normal_bf16(1201, 0, (M, K)), I.normal_bf16(1202, 0, (M, N))
    want = vc.vitcop_project_mx4(dev(x), codes, scales, residual=dev(r))
    y = dev(r)
    assert torch.equal(vc.vitcop_project_mx4(dev(x), codes, scales, residual=y, out=y), want)
    scales[5, 3] = 255                                                    # a group of row 5: column 5 of every output row
    got = vc.vitcop_project_mx4(dev(x), codes, scales, residual=dev(r))
    assert torch.isnan(got[:, 5]).all() and torch.equal(got[:, 6:], want[:, 6:]) and torch.equal(got[:, :5], want[:, :5])
    x[4, 17] = 0x7FC0                                                     # a value of x's row 4: that row
    got = vc.vitcop_project_mx4(dev(x), *vc.vitcop_mx4_quantize(dev(w)), residual=dev(r))
    assert torch.isnan(got[4]).all() and torch.equal(got[5:], want[5:]) and torch.equal(got[:4], want[:4])


def test_equal_rows_have_equal_results(vc):
    # wherever they stand among up to 64 rows, and from call to call
    K, N = 1056, 80
    row = I.normal_bf16(1300, 0, (1, K))
    for M in (1, 16, 40, 64, 150):
        y = project_check(vc, M, N, K, False, seed=5, x=np.repeat(row, M, 0))
        assert all(torch.equal(y[m], y[0]) for m in range(M))
    row = I.normal_bf16(1301, 0, (1, 4096))
    for M in (50, 170):
        y = project_check(vc, M, 4096, 4096, False, seed=6, x=np.repeat(row, M, 0))
        assert all(torch.equal(y[m], y[0]) for m in range(M))


# ----------------------------------------------------------------------------------------- used together


def decode_layer(vc, h, w4, ln1, ln2, cache, n_cached, N, positions, Hq, Hkv, d):
    """One token per sample through a layer whose weights and cache are held in 4 bits: what a program composes."""
    B = h.shape[0]
    a = vc.vitcop_rmsnorm(h, ln1)
    q, k, v = (vc.vitcop_project_mx4(a, *w4[n]) for n in ("wq", "wk", "wv"))
    q, k, v = q.view(B, 1, Hq, d), k.view(B, 1, Hkv, d), v.view(B, 1, Hkv, d)
    vc.vitcop_rope(q, k, positions)
    vc.vitcop_cache_mx4_write(cache, k, v, start_samples=n_cached)
    o, _ = vc.vitcop_decode_attn_mx4(q.view(B, Hq, d), cache, N, n_samples=n_cached + 1, want_lse=False)
    h1 = vc.vitcop_project_mx4(o.view(B, Hq * d), *w4["wo"], residual=h)
    b = vc.vitcop_rmsnorm(h1, ln2)
    act = vc.vitcop_silu_mul(vc.vitcop_project_mx4(b, *w4["wg"]), vc.vitcop_project_mx4(b, *w4["wu"]))
    return {"a": a, "q": q, "k": k, "v": v, "o": o, "h1": h1, "b": b, "act": act,
            "y": vc.vitcop_project_mx4(act, *w4["wd"], residual=h1)}


def layer_setup(vc, B, D, Hq, Hkv, d, F, T, capacity):
    c = I.decoder_inputs(1400, B, T, D, Hq, Hkv, d, F)
    w = c["w"]
    wd = {n: dev(x) for n, x in w.items()}
    w4 = {n: vc.vitcop_mx4_quantize(wd[n]) for n in w if n[0] == "w"}
    return c, w, wd, w4


def test_prefill_then_decoding_in_4_bits(vc):
    # a pruned prefill leaves a bf16 cache; it is held in 4 bits from there on, and three tokens are decoded over it, every
    # stage against the oracle on the stage's own inputs
    B, T, D, Hq, Hkv, d, F, vs, nv, keep = 3, 120, 256, 4, 2, 64, 384, 8, 80, 20
    c, w, wd, w4 = layer_setup(vc, B, D, Hq, Hkv, d, F, T, 80)
    Tp = T - nv + keep
    kc, vcache = (torch.zeros((B, 70, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda").repeat(B, 1)
    vc.vitcop_decoder_layer_prefill(dev(c["h"]), pos, wd, Hq, Hkv, d, vs, nv, keep, caches=(kc, vcache))
    cache = vc.CacheMx4.empty(B, 80, Hkv, d)
    counts = [Tp, Tp - 7, 33]
    vc.vitcop_cache_mx4_write(cache, kc[:, :Tp], vcache[:, :Tp], n_samples=i32(counts))
    kv = contents(cache)
    for b in range(B):
        for side, x in ((0, kc), (1, vcache)):
            assert np.array_equal(kv[side][b, :, :counts[b]], X.round_trip(host_bits(x))[b, :counts[b]].transpose(1, 0, 2))
    h = dev(I.normal_bf16(1401, 0, (B, D)))
    for step in range(3):
        n = [x + step for x in counts]
        positions = i32([[T + step]] * B)
        s = decode_layer(vc, h, w4, wd["ln1"], wd["ln2"], cache, i32(n), max(n) + 1, positions, Hq, Hkv, d)
        g = {k: host_bits(t) for k, t in s.items()}

        def product(x, name, res=None):
            xv, wv = O.bf16_to_f64(x), X.round_trip(w[name])
            ref, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
            return (ref, size) if res is None else (ref + O.bf16_to_f64(res), size + np.abs(O.bf16_to_f64(res)))

        def near(got, ref, size, n_sum, what):
            assert (np.abs(O.bf16_to_f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + (n_sum + 4) * EPS * size).all(), what

        near(g["v"].reshape(B, -1), *product(g["a"], "wv"), D, "v")
        near(g["h1"], *product(g["o"].reshape(B, -1), "wo", host_bits(h)), Hq * d, "h1")
        near(g["y"], *product(g["act"], "wd", g["h1"]), F, "y")
        # a gate and an up value are each rounded before the product of the two: three half steps, and the sums' own error
        gate, gs = product(g["b"], "wg")
        up, us = product(g["b"], "wu")
        act = gate / (1 + np.exp(-gate)) * up
        off = 1.2 * (2.0 ** -8 * np.abs(gate) + (D + 4) * EPS * gs) * np.abs(up) + \
            np.abs(gate / (1 + np.exp(-gate))) * (2.0 ** -8 * np.abs(up) + (D + 4) * EPS * us)
        assert (np.abs(O.bf16_to_f64(g["act"]) - act) <= 2.0 ** -8 * np.abs(act) + 1.02 * off + 1e-30).all()
        after = contents(cache)
        for b in range(B):
            for side, x in ((0, g["k"]), (1, g["v"])):
                kv[side][b, :, n[b]] = X.round_trip(x)[b, 0]
                assert np.array_equal(after[side][b, :, :n[b] + 1], kv[side][b, :, :n[b] + 1])
        kv = after
        ref, _, spread, size = X.decode_attention(g["q"][:, 0], kv[0], kv[1], [x + 1 for x in n])
        p_off = (d + 4) * EPS * size + 2.0 ** -16 + 2.0 ** -20 + 80 * EPS
        assert (np.abs(O.bf16_to_f64(g["o"]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * p_off[..., None] * spread).all()
        h = s["y"]


def test_captured_and_on_another_stream(vc):
    # the layer's calls recorded into a graph and replayed among eager calls, and eagerly on a stream of its own
    B, D, Hq, Hkv, d, F = 2, 256, 4, 2, 64, 384
    c, w, wd, w4 = layer_setup(vc, B, D, Hq, Hkv, d, F, 300, 301)
    t = I.qkv_tensors(1500, B, 300, Hq, Hkv, d)
    cache = vc.CacheMx4.empty(B, 301, Hkv, d)
    vc.vitcop_cache_mx4_write(cache, dev(t["k"]), dev(t["v"]))
    n, positions = i32([300, 150]), i32([[300]] * B)
    hs = [dev(I.normal_bf16(1501 + i, 0, (B, D))) for i in range(4)]
    layer = lambda x: decode_layer(vc, x, w4, wd["ln1"], wd["ln2"], cache, n, 301, positions, Hq, Hkv, d)["y"]  # noqa: E731
    want = [layer(x).clone() for x in hs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [layer(x) for x in hs]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    h = hs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer(h)
    for i in (1, 2, 3, 0):
        h.copy_(hs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
        assert torch.equal(layer(hs[i]), want[i])


def test_two_graphs_of_calls_with_workspaces(vc):
    # sliced attention, a sliced projection and one by way of bf16, in two graphs on inputs of their own, replayed in turn and
    # at once on two streams, with eager calls between
    B, N, Hq, Hkv, d = 3, 2000, 8, 2, 128
    t = I.qkv_tensors(1600, B, N, Hq, Hkv, d)
    cache = vc.CacheMx4.empty(B, N, Hkv, d)
    vc.vitcop_cache_mx4_write(cache, dev(t["k"]), dev(t["v"]))
    matrices = [vc.vitcop_mx4_quantize(dev(I.normal_bf16(1601, i, shape, std=0.02)))
                for i, shape in enumerate([(640, 4448), (4096, 256)])]
    rows = (316, 700)
    assert vc.lib.vitcop_decode_attn_mx4_workspace_bytes(B, N, Hq, Hkv, d) > 0
    assert all(vc.lib.vitcop_project_mx4_workspace_bytes(m, c.shape[0], 2 * c.shape[1]) > 0 for m, (c, _) in zip(rows, matrices))

    def calls(q, xs):
        return [vc.vitcop_decode_attn_mx4(q, cache, N)[0]] + [vc.vitcop_project_mx4(x, *w) for x, w in zip(xs, matrices)]

    inputs = [(dev(I.normal_bf16(1610 + i, 0, (B, Hq, d))),
               [dev(I.normal_bf16(1620 + i, j, (m, 2 * matrices[j][0].shape[1]))) for j, m in enumerate(rows)]) for i in range(2)]
    want = [[y.clone() for y in calls(*x)] for x in inputs]
    graphs, outputs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for x in inputs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outputs.append(calls(*x))
    torch.cuda.synchronize()
    for turn in range(4):
        for g, side in zip(graphs, streams):
            if turn % 2 == 0:
                g.replay()
            else:
                with torch.cuda.stream(side):
                    g.replay()
        eager = calls(*inputs[turn % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for got, ref in zip(outputs, want) for a, b in zip(got, ref)), turn
        assert all(torch.equal(a, b) for a, b in zip(eager, want[turn % 2])), turn


def test_the_binding_refuses(vc):
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    codes, scales = vc.vitcop_mx4_quantize(x)
    cache = vc.CacheMx4.empty(2, 8, 2, 64)
    rows = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: vc.vitcop_mx4_quantize(x.half()), lambda: vc.vitcop_cache_mx4_write(cache, rows.half(), None),
                lambda: vc.vitcop_decode_attn_mx4(q.half(), cache, 8), lambda: vc.vitcop_project_mx4(x.half(), codes, scales),
                lambda: vc.vitcop_mx4_dequantize(codes[0], scales), lambda: vc.vitcop_project_mx4(x, codes[0], scales),
                lambda: vc.vitcop_mx4_quantize(x.float()), lambda: vc.vitcop_mx4_quantize(x.t()),
                lambda: vc.vitcop_mx4_dequantize(codes, scales[:3]), lambda: vc.vitcop_mx4_dequantize(codes.cpu(), scales),
                lambda: vc.vitcop_mx4_dequantize(codes, scales, out=x[:3]),
                lambda: vc.CacheMx4(cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales[:1]),
                lambda: vc.CacheMx4(cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales.char()),
                lambda: vc.vitcop_cache_mx4_write(cache, rows, rows[:, :2]),
                lambda: vc.vitcop_cache_mx4_write(cache, rows[:1], rows[:1]),
                lambda: vc.vitcop_cache_mx4_write(cache, rows.transpose(2, 3), None),
                lambda: vc.vitcop_cache_mx4_write(cache, rows.cpu(), None),
                lambda: vc.vitcop_cache_mx4_write(cache, rows, rows, start_samples=torch.zeros(2, device="cuda")),
                lambda: vc.vitcop_cache_mx4_write(cache, rows, rows, n_samples=i32([1])),
                lambda: vc.vitcop_cache_mx4_read(cache, -1),
                lambda: vc.vitcop_cache_mx4_read(cache, 2, out=(rows, rows)),
                lambda: vc.vitcop_decode_attn_mx4(q[:1], cache, 8), lambda: vc.vitcop_decode_attn_mx4(q.transpose(0, 1), cache, 8),
                lambda: vc.vitcop_decode_attn_mx4(q, cache, 8, n_samples=i32([1, 1, 1])),
                lambda: vc.vitcop_decode_attn_mx4(q, cache, 8, ws=torch.zeros(1 << 20, device="cuda")),
                lambda: vc.vitcop_project_mx4(x[:, :32], codes, scales), lambda: vc.vitcop_project_mx4(x, codes.t(), scales),
                lambda: vc.vitcop_project_mx4(x, codes, scales, residual=x)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: vc.vitcop_cache_mx4_write(cache, rows, rows, start=6),
                lambda: vc.vitcop_cache_mx4_read(cache, 9), lambda: vc.vitcop_decode_attn_mx4(q, cache, 9),
                lambda: vc.vitcop_project_mx4(x, codes, scales), lambda: vc.vitcop_mx4_quantize(x[:, :40])):
        with pytest.raises(vc.VitcopError):
            bad()
