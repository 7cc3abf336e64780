"""CPU oracle for values held in 4 bits and the decoding over them, in NumPy float64.  TEST INFRASTRUCTURE ONLY.

Groups of 32 values share an exponent byte s; a value is code * 2^(s - 127), a code a sign and one of the eight magnitudes
below.  The exponent is the least in [-125, 125] that leaves no magnitude above 7 steps, the code the nearest value, ties to
the even code.  A group with an infinity or a NaN has s = 255 and stands for NaN.
"""
from __future__ import annotations

import numpy as np

from . import vitcop_oracle as O

GROUP = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(bits):
    """bf16 bits [..., K] -> (codes [..., K/2], scales [..., K/32]) uint8."""
    x = O.bf16_to_f64(bits)
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    e = np.full(top.shape, -125)
    while True:                                      # the definition, one exponent at a time
        low = (top > 7.0 * np.exp2(e.astype(np.float64))) & (e < 125)
        if not low.any():
            break
        e[low] += 1
    t = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    off = np.abs(t[..., None] - MAGNITUDES)
    near = off == off.min(-1, keepdims=True)
    even = np.arange(8) % 2 == 0
    code = np.where((near & even).any(-1), (near & even).argmax(-1), near.argmax(-1))    # two at a tie: one of them is even
    code = (code + 8 * np.signbit(g)).astype(np.uint8).reshape(x.shape)
    code[np.repeat(~finite, GROUP, -1).reshape(x.shape)] = 0
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def values(codes, scales) -> np.ndarray:
    """What codes [..., K/2] and scales [..., K/32] stand for, float64 [..., K]."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    step = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return v * np.repeat(step, GROUP, -1)


def round_trip(bits) -> np.ndarray:
    return values(*quantize(bits))


def decode_attention(q_bits, k, v, lens=None, scale: float | None = None):
    """q [B,Hq,d] bits, k, v float64 [B,Hkv,N,d] -> (out [B,Hq,d], lse [B,Hq], spread [B,Hq,d], size [B,Hq]):
    sample b attends over its first lens[b] rows (without any: 0 and -inf).  For error bounds: spread = sum_j p_j |v_j|,
    size = max_j scale * sum_c |q_c k_jc|."""
    q = O.bf16_to_f64(q_bits)
    B, Hq, d = q.shape
    G = Hq // k.shape[1]
    scale = 1.0 / np.sqrt(d) if not scale else scale
    out, spread = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    lse, size = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    for b in range(B):
        n = k.shape[2] if lens is None else int(lens[b])
        for h in range(Hq if n else 0):
            kk, vv = k[b, h // G, :n], v[b, h // G, :n]
            s = kk @ q[b, h] * scale
            top = s.max()
            p = np.exp(s - top)
            lse[b, h] = top + np.log(p.sum())
            p /= p.sum()
            out[b, h], spread[b, h] = p @ vv, p @ np.abs(vv)
            size[b, h] = (np.abs(kk) @ np.abs(q[b, h])).max() * scale
    return out, lse, spread, size
