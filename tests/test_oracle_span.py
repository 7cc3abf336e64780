"""Pins of the oracle of the calls on prompts, tokens and drafts over a bf16 cache: library functions, closed forms, and what is
known of the forms that it has to agree with."""
import math

import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import decoder_oracle as D
from oracle import span_oracle as S
from oracle import vitcop_oracle as O


def test_axes_of_pairs():
    assert S.axis_of_pairs((2, 1, 3), False) == [0, 0, 1, 2, 2, 2]
    assert S.axis_of_pairs((2, 1, 3), True) == [0, 1, 2, 0, 2, 2]
    assert S.axis_of_pairs((0, 2), True) == [1, 1]


def test_revolutions_against_floats():
    pos = np.arange(-40, 60).reshape(1, 2, 50)
    want = pos[0][:, :, None] * 10000.0 ** (-2.0 * np.arange(32) / 64) / (2 * math.pi)
    got = S.revolutions(pos, (32,), 10000.0)
    off = got - want
    assert np.abs(off - np.round(off)).max() < 1e-12 and (np.abs(got) <= 0.5).all()


def test_far_positions_add_up():
    # the angle of a sum is the sum of the angles, at any distance
    a, b = 2 ** 31 - 1, -2 ** 31
    t = S.revolutions(np.array([[[a, b, a + b]]]), (8,), 1e6)[0]
    off = t[0] + t[1] - t[2]
    assert np.abs(off - np.round(off)).max() < 1e-12


def test_one_axis_is_the_rotary_embedding_of_the_decoder():
    rng = np.random.default_rng(0)
    bits = I.f32_to_bf16_bits(rng.standard_normal((2, 5, 3, 32)).astype(np.float32))
    pos = rng.integers(0, 500, (2, 5))
    got = S.rope_axes(O.bf16_to_f64(bits), S.revolutions(np.stack([pos, pos]), (9, 7), 10000.0, True))
    assert np.abs(got - D.rope(bits, pos, 10000.0)).max() < 1e-10


def test_axes_turn_their_own_pairs():
    x = np.ones((1, 1, 1, 8))
    y = S.rope_axes(x, S.revolutions(np.array([[[0]], [[7]]]), (2, 2), 100.0))[0, 0, 0]
    assert np.array_equal(y[[0, 1, 4, 5]], np.ones(4))                       # position 0: not turned
    speed = 100.0 ** (-2 * 3 / 8)
    assert abs(y[3] - (math.cos(7 * speed) - math.sin(7 * speed))) < 1e-12


def test_without_a_window_it_is_causal_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((7, 4, 64)), rng.standard_normal((7, 2, 64)), rng.standard_normal((7, 2, 64))
    want = torch.nn.functional.scaled_dot_product_attention(
        *[torch.from_numpy(x).transpose(0, 1) for x in (q, k.repeat(2, 1), v.repeat(2, 1))], is_causal=True)
    got = S.attend(q, k, v, S.window_sees(0, 7, 7, 0, 0))
    assert np.abs(got["out"] - want.transpose(0, 1).numpy()).max() < 1e-12


def test_windows_by_hand():
    assert S.window_sees(3, 2, 6, 2, 1).astype(int).tolist() == [[1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0]]
    assert S.window_sees(0, 2, 3, 1, 0).astype(int).tolist() == [[1, 0, 0], [0, 1, 0]]
    assert S.window_sees(0, 2, 2, 1, 9).astype(int).tolist() == [[1, 0], [1, 1]]       # a sink is no sooner seen than written


def test_trees_by_hand():
    assert S.tree_sees(2, 3, [0b001, 0b011, 0b101]).astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 0, 1]]
    assert S.tree_sees(0, 1, [-2 ** 63]).astype(int).tolist() == [[0]]
    far = S.tree_sees(0, 64, [2 ** 64 - 1, 1] + [1 << 63 | 1 << 9] * 62).astype(int)     # (64 bits, not 53)
    assert far.sum(1).tolist() == [64, 1] + [2] * 62 and far[5, 9] == far[63, 63] == 1


def test_nothing_seen():
    r = S.attend(np.ones((1, 2, 64)), np.ones((3, 1, 64)), np.ones((3, 1, 64)), np.zeros((1, 3), bool))
    assert not r["out"].any() and (r["lse"] == -math.inf).all()


@pytest.mark.parametrize("scale", [0.0, 0.3])
def test_lse_against_scipy(scale):
    from scipy.special import logsumexp
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 1, 64)), rng.standard_normal((9, 1, 64)), rng.standard_normal((9, 1, 64))
    sees = rng.random((3, 9)) < 0.5
    sees[:, 0] = True
    r = S.attend(q, k, v, sees, scale)
    s = np.where(sees, q[:, 0] @ k[:, 0].T * (scale or 0.125), -math.inf)
    assert np.abs(r["lse"][0] - logsumexp(s, 1)).max() < 1e-12
    assert (r["mass"] >= np.abs(r["out"]) - 1e-12).all() and (r["reach"][:, 0] >= s.max(1)).all()
