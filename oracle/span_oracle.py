"""CPU oracle of the calls on prompts, tokens and drafts over a bf16 cache, from their definitions: rotary positions of several
axes in whole revolutions of 128 bits, attention in float64 over an explicit mask."""
from __future__ import annotations

import decimal
import math

import numpy as np

_PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def axis_of_pairs(sections, interleaved):
    """The axis of each pair: section after section, or a pair to each axis in turn while it has one left."""
    if not interleaved:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return out


def revolutions(positions, sections, theta, interleaved=False):
    """positions [n_axes,B,T] -> the angle of each pair as a part of a revolution in [-1/2, 1/2), [B,T,d/2] float64."""
    axis = axis_of_pairs(sections, interleaved)
    half = len(axis)
    with decimal.localcontext() as ctx:
        ctx.prec = 70
        log = decimal.Decimal(float(theta)).ln()
        speed = [int((-log * i / half).exp() / (2 * _PI) * 2 ** 128) for i in range(half)]
    n_axes, B, T = positions.shape
    out = np.empty((B, T, half))
    for i, (a, s) in enumerate(zip(axis, speed)):
        for b in range(B):
            for t in range(T):
                turn = int(positions[a, b, t]) * s % 2 ** 128
                out[b, t, i] = (turn - 2 ** 128 if turn >= 2 ** 127 else turn) / 2.0 ** 128
    return out


def rope_axes(x, turns):
    """x [B,T,H,d] float64 turned by turns [B,T,d/2] (in revolutions): pairs (i, i + d/2)."""
    half = x.shape[-1] // 2
    c, s = np.cos(2 * math.pi * turns)[:, :, None], np.sin(2 * math.pi * turns)[:, :, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def window_sees(start, n, keys, window, sinks):
    """[n,keys]: token t at row start + t sees row j."""
    row, j = start + np.arange(n)[:, None], np.arange(keys)
    near = (j > row - window) | (j < sinks) if window else True
    return (j <= row) & near


def tree_sees(start, n, masks):
    """[n, start + n]: all of the cache's rows, and the drafts whose bit is set."""
    bits = (np.array([int(m) % 2 ** 64 for m in masks[:n]], np.uint64)[:, None] >> np.arange(n, dtype=np.uint64)) & np.uint64(1)
    return np.concatenate([np.ones((n, start), bool), bits.astype(bool)], 1)


def attend(q, k, v, sees, scale=0.0):
    """q [n,Hq,d], k, v [N,Hkv,d], sees [n,N] -> dict of out [n,Hq,d], lse [Hq,n] and what bounds an error: mass [n,Hq,d], the
    sum of p |v|, and reach [n,Hq], the largest sum of |q k| scale among the keys that are seen."""
    n, Hq, d = q.shape
    Hkv = k.shape[1]
    scale = scale or 1.0 / math.sqrt(d)
    r = dict(out=np.zeros((n, Hq, d)), lse=np.full((Hq, n), -math.inf), mass=np.zeros((n, Hq, d)), reach=np.zeros((n, Hq)))
    rows = np.flatnonzero(sees.any(0))
    if n == 0 or len(rows) == 0:
        return r
    sees = sees[:, rows]
    for h in range(Hq):
        kh, vh = k[rows, h // (Hq // Hkv)], v[rows, h // (Hq // Hkv)]
        s = np.where(sees, q[:, h] @ kh.T * scale, -math.inf)
        top = s.max(1)
        some = np.isfinite(top)
        p = np.where(sees, np.exp(s - np.where(some, top, 0.0)[:, None]), 0.0)
        total = p.sum(1)
        w = p / np.where(some, total, 1.0)[:, None]
        r["out"][:, h], r["mass"][:, h] = w @ vh, w @ np.abs(vh)
        r["lse"][h] = np.where(some, np.log(np.where(some, total, 1.0)) + np.where(some, top, 0.0), -math.inf)
        r["reach"][:, h] = np.where(sees, np.abs(q[:, h]) @ np.abs(kh).T * scale, 0.0).max(1)
    return r
