"""Pins for the oracle of values held in 4 bits."""
import numpy as np
import pytest

import vitcop_inputs as I
from oracle import mx4_oracle as X
from oracle import vitcop_oracle as O


def bits(a):
    return I.f32_to_bf16_bits(np.asarray(a, dtype=np.float32))


def test_every_code_of_a_group_reads_back_as_itself():
    g = np.zeros(32)
    g[:16] = np.concatenate([X.MAGNITUDES, -X.MAGNITUDES])
    codes, scales = X.quantize(bits(g * 8))
    assert scales.tolist() == [130] and codes[:8].tolist() == [0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE]
    assert np.array_equal(X.values(codes, scales), g * 8)


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (0.26, 1), (0.74, 1),
                                    (1.26, 3), (2.51, 5), (3.49, 5), (5.03, 7), (6.5, 7), (7.0, 7)])
def test_nearest_code_and_ties(x, code):
    g = np.zeros(32)
    g[0], g[1], g[2] = x, -x, 4.0                     # (4: the group's exponent is 0 whatever x is)
    codes, scales = X.quantize(bits(g))
    assert scales[0] == 127 and codes[0] == code + 16 * (code + 8) and codes[1] == 6


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.03125, 1), (3.5, -1), (3.515625, 0), (1e-45, -125), (0.0, -125),
                                   (7 * 2.0 ** -125, -125), (7.03125 * 2.0 ** -125, -124), (3.3e38, 125), (2.5e38, 125)])
def test_exponent(top, e):
    g = np.zeros(32)
    g[31] = -top
    assert X.quantize(bits(g))[1][0] == e + 127


def test_error_is_at_most_one_step_and_half_below_four():
    x = I.normal_bf16(1, 0, (64, 256))
    codes, scales = X.quantize(x)
    f, v = O.bf16_to_f64(x), X.values(codes, scales)
    step = np.repeat(np.exp2(scales.astype(float) - 127), 32, -1)
    off = np.abs(f - v) / step
    assert off.max() <= 1.0 and off[np.abs(f) < 4 * step].max() <= 0.5 and off[np.abs(f) < 2 * step].max() <= 0.25
    assert np.array_equal(np.signbit(f), np.signbit(v))
    assert np.array_equal(X.round_trip(O.f64_to_bf16_bits(v)), v)        # what is held is held again as it is


def test_a_group_that_is_not_finite():
    x = I.normal_bf16(2, 0, (1, 96)).copy()
    x[0, 40], x[0, 95] = 0x7F80, 0x7FC1
    v = X.round_trip(x)
    assert np.isfinite(v[0, :32]).all() and np.isnan(v[0, 32:]).all()


def test_decode_attention_is_the_other_oracles():
    from oracle import decoder_oracle as Dc
    t = I.qkv_tensors(3, 2, 37, 6, 2, 64)
    k, v = (O.bf16_to_f64(t[n]).transpose(0, 2, 1, 3) for n in ("k", "v"))
    out, lse, _, _ = X.decode_attention(t["q"][:, -1], k, v)
    ref, ref_lse = Dc.decode_attention(t["q"][:, -1], t["k"], t["v"])
    assert np.allclose(out, ref, rtol=1e-12, atol=1e-14) and np.allclose(lse, ref_lse, rtol=1e-12)
    out, lse, _, _ = X.decode_attention(t["q"][:, -1], k, v, lens=[0, 5])
    ref, _ = Dc.decode_attention(t["q"][1:, -1], t["k"][1:, :5], t["v"][1:, :5])
    assert not out[0].any() and np.isneginf(lse[0]).all() and np.allclose(out[1:], ref, rtol=1e-12)
