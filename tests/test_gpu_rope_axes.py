"""vitcop_rope_axes and vitcop_cache_append: turned rows against angles of 128 bits, moved rows bit for bit.

Bound of a turned value y = x c - z s: the angle's fraction of a revolution goes to fp32 (relative 2^-24 of at most pi), sine
and cosine are off by 2^-23, three fp32 roundings: together below 2^-20 (|x| + |z|), and the rounding to bf16, 2^-8 |y|.
"""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from gpu_util import dev, host_bits, host_f64
from oracle import span_oracle as S
from oracle import vitcop_oracle as O

pytestmark = pytest.mark.gpu

MARK = 0x40F0                  # 7.5


@pytest.fixture(scope="module")
def vc():
    from paper_2601_17818_amd import binding
    return binding


def bits(rng, shape):
    return I.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def marked(shape):
    return dev(np.full(shape, MARK, np.uint16))


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def assert_turned(got, x_bits, turns, where):
    x = O.bf16_to_f64(x_bits)
    want = S.rope_axes(x, turns)
    half = x.shape[-1] // 2
    mates = np.abs(x) + np.abs(np.concatenate([x[..., half:], x[..., :half]], -1))
    err = np.abs(O.bf16_to_f64(got) - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * mates).all(), (where, err.max())


SIZES = [
    # B, T, Hq, Hkv, d, sections, interleaved
    (1, 1, 28, 4, 128, (16, 24, 24), False), (2, 3, 4, 2, 64, (8, 12, 12), True), (3, 1, 1, 1, 16, (8,), False),
    (1, 5, 3, 1, 48, (5, 19), True), (2, 7, 2, 2, 256, (32, 32, 32, 32), True), (1, 2, 5, 5, 80, (0, 40, 0), False),
    (1, 700, 8, 8, 128, (24, 20, 20), True), (2, 333, 16, 4, 64, (10, 11, 11), False), (1, 4100, 12, 2, 128, (16, 24, 24), False)]


@pytest.mark.parametrize("B,T,Hq,Hkv,d,sections,interleaved", SIZES)
def test_against_the_oracle(vc, B, T, Hq, Hkv, d, sections, interleaved):
    rng = np.random.default_rng(T)
    q, k = bits(rng, (B, T, Hq, d)), bits(rng, (B, T, Hkv, d))
    pos = rng.integers(-50, 40000, (len(sections), B, T)).astype(np.int32)
    some = min(T, 400)                                   # (the oracle's exact angles take their time)
    pos[:, :, some:] = pos[:, :, :1]
    qo, ko = vc.vitcop_rope_axes(dev(q), dev(k), ints(pos), sections, 1000000.0, interleaved=interleaved)
    turns = S.revolutions(pos[:, :, :some], sections, 1000000.0, interleaved)
    turns = np.concatenate([turns, np.repeat(turns[:, :1], T - some, 1)], 1)
    assert_turned(host_bits(qo), q, turns, "q")
    assert_turned(host_bits(ko), k, turns, "k")


def test_far_positions(vc):
    rng = np.random.default_rng(1)
    q = bits(rng, (1, 6, 2, 128))
    pos = np.array([[[2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 10 ** 9, -1, 0]]], np.int32)
    qo, ko = vc.vitcop_rope_axes(dev(q), None, ints(pos), (64,), 10000.0)
    assert ko is None
    assert_turned(host_bits(qo), q, S.revolutions(pos, (64,), 10000.0), "q")


def test_one_axis_is_vitcop_rope(vc):
    rng = np.random.default_rng(2)
    q, k = bits(rng, (2, 9, 4, 128)), bits(rng, (2, 9, 2, 128))
    pos = ints(rng.integers(0, 600, (2, 9)))
    qo, ko = vc.vitcop_rope_axes(dev(q), dev(k), pos[None], (64,))
    qr, kr = vc.vitcop_rope(dev(q), dev(k), pos)
    for a, b in ((qo, qr), (ko, kr)):                    # (its angles are fp32: 600 x 2^-23 beside half a step each)
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()


@pytest.mark.parametrize("T,counts", [(1, None), (6, [6, 0, 2]), (400, [400, 399, 1])])
def test_into_a_cache(vc, T, counts):
    """Fused rows to a buffer of queries and the cache's rows; everything else stays as it was."""
    B, Hq, Hkv, d, capacity = 3, 8, 2, 128, T + 9
    rng = np.random.default_rng(3)
    rows = bits(rng, (B, T + 1, (Hq + 2 * Hkv), d))
    fused = dev(rows)[:, :T]
    q, k, v = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:]
    pos = rng.integers(0, 3000, (3, B, T)).astype(np.int32)
    start = np.array([9, 0, 4])
    kc, vcache, out = marked((B, capacity, Hkv, d)), marked((B, capacity, Hkv, d)), marked((B, T, Hq, d))
    cache = vc.Cache(kc, vcache)
    got, none = vc.vitcop_rope_axes(q, k, ints(pos), (16, 24, 24), v=v, cache=cache, start_samples=ints(start),
                                    n_samples=ints(counts) if counts else None, out=out)
    assert got is out and none is None
    turns = S.revolutions(pos, (16, 24, 24), 10000.0)
    for b in range(B):
        n, s = (counts[b] if counts else T), start[b]
        x = rows[b, :T]
        assert_turned(host_bits(out)[b, :n], x[:n, :Hq], turns[b:b + 1, :n], f"q {b}")
        assert (host_bits(out)[b, n:] == MARK).all()
        assert_turned(host_bits(kc)[b, s:s + n], x[:n, Hq:Hq + Hkv], turns[b:b + 1, :n], f"k {b}")
        assert np.array_equal(host_bits(vcache)[b, s:s + n], x[:n, Hq + Hkv:])
        for c in (kc, vcache):
            left = host_bits(c)[b]
            assert (left[:s] == MARK).all() and (left[s + n:] == MARK).all()


def test_rows_outside_the_cache_are_skipped(vc):
    B, T, Hkv, d, capacity = 4, 3, 2, 64, 5
    rng = np.random.default_rng(4)
    k, v = bits(rng, (B, T, Hkv, d)), bits(rng, (B, T, Hkv, d))
    kc, vcache = marked((B, capacity, Hkv, d)), marked((B, capacity, Hkv, d))
    start = [-1, 4, 2 ** 31 - 1, -2 ** 31]
    pos = np.zeros((2, B, T), np.int32)
    q, _ = vc.vitcop_rope_axes(None, dev(k), ints(pos), (20, 12), v=dev(v), cache=vc.Cache(kc, vcache), start_samples=ints(start))
    assert q is None
    want_k, want_v = np.full((B, capacity, Hkv, d), MARK, np.uint16), np.full((B, capacity, Hkv, d), MARK, np.uint16)
    for b in range(B):
        for t in range(T):
            if 0 <= start[b] + t < capacity:
                want_k[b, start[b] + t], want_v[b, start[b] + t] = k[b, t], v[b, t]
    assert np.array_equal(host_bits(kc), want_k) and np.array_equal(host_bits(vcache), want_v)


def test_values_alone_outside_the_cache_are_skipped(vc):
    B, T, Hkv, d, capacity = 3, 2, 2, 64, 4
    rng = np.random.default_rng(9)
    v = bits(rng, (B, T, Hkv, d))
    room = marked((B + 2, capacity, Hkv, d))                             # (the cache lies between two more)
    cache = vc.Cache(marked((B, capacity, Hkv, d)), room[1:B + 1])
    vc.vitcop_rope_axes(None, None, ints(np.zeros((1, B, T))), (32,), v=dev(v), cache=cache, start_samples=ints([-1, 3, 4]))
    want = np.full((B + 2, capacity, Hkv, d), MARK, np.uint16)
    want[1, 0], want[2, 3] = v[0, 1], v[1, 0]
    assert np.array_equal(host_bits(room), want)


def test_in_place_and_values_alone(vc):
    B, T, H, d = 2, 11, 3, 64
    rng = np.random.default_rng(5)
    rows = bits(rng, (B, T, 3 * H, d))
    pos = rng.integers(0, 900, (2, B, T)).astype(np.int32)
    turns = S.revolutions(pos, (30, 2), 10000.0, True)
    fused = dev(rows)
    q, k = fused[:, :, :H], fused[:, :, H:2 * H]
    qo, ko = vc.vitcop_rope_axes(q, k, ints(pos), (30, 2), interleaved=True, out=q, k_out=k)
    assert qo is q and ko is k
    assert_turned(host_bits(q), rows[:, :, :H], turns, "q")
    assert_turned(host_bits(k), rows[:, :, H:2 * H], turns, "k")
    assert np.array_equal(host_bits(fused[:, :, 2 * H:]), rows[:, :, 2 * H:])
    cache = vc.Cache(marked((B, T, H, d)), marked((B, T, H, d)))
    vc.vitcop_rope_axes(None, None, ints(pos), (30, 2), v=fused[:, :, 2 * H:], cache=cache)
    assert np.array_equal(host_bits(cache.v), rows[:, :, 2 * H:]) and (host_bits(cache.k) == MARK).all()


def appended(caches, k, starts, idx, counts):
    out = [c.copy() for c in caches]
    for layer in range(len(caches)):
        B, capacity = caches[layer].shape[:2]
        for b in range(B):
            rows = idx.shape[1] if idx is not None else k.shape[2]
            for i in range(min(max(counts[b], 0), rows) if counts is not None else rows):
                src, to = (int(idx[b, i]) if idx is not None else i), int(starts[layer][b]) + i
                if 0 <= src < k.shape[2] and 0 <= to < capacity:
                    out[layer][b, to] = k[layer, b, src]
    return out


@pytest.mark.parametrize("L,B,T,rows,Hkv,d,capacity", [(1, 1, 1, 1, 1, 64, 1), (3, 2, 8, 4, 2, 128, 30), (70, 2, 5, 3, 1, 64, 9),
                                                        (2, 3, 64, 12, 4, 128, 200), (2, 2, 300, 300, 3, 40, 400)])
@pytest.mark.parametrize("stacked", [True, False])
def test_append(vc, L, B, T, rows, Hkv, d, capacity, stacked):
    rng = np.random.default_rng(6)
    k, v = bits(rng, (L, B, T, Hkv, d)), bits(rng, (L, B, T, Hkv, d))
    kc, vcache = bits(rng, (L, B, capacity, Hkv, d)), bits(rng, (L, B, capacity, Hkv, d))
    starts = rng.integers(-2, capacity + 1, (L, B))
    idx = rng.integers(0, T, (B, rows))
    idx[0, -1] = rng.choice([idx[0, 0], T, -1, 2 ** 31 - 1])             # twice the same, or none that there is
    counts = rng.integers(0, rows + 2, B)
    kd, vd = dev(kc), dev(vcache)
    views = (kd, vd) if stacked else (list(kd), list(vd))
    wide = dev(np.concatenate([k, v, k], -2))                            # k and v in fused rows
    vc.vitcop_cache_append(*views, wide[:, :, :, :Hkv], wide[:, :, :, Hkv:2 * Hkv], start_samples=ints(starts), idx=ints(idx),
                           n_samples=ints(counts))
    assert np.array_equal(host_bits(kd), np.stack(appended(kc, k, starts, idx, counts)))
    assert np.array_equal(host_bits(vd), np.stack(appended(vcache, v, starts, idx, counts)))


def test_append_without_paths(vc):
    L, B, T, Hkv, d, capacity = 2, 2, 6, 2, 64, 20
    rng = np.random.default_rng(7)
    k = bits(rng, (L, B, T, Hkv, d))
    kc = bits(rng, (L, B, capacity, Hkv, d))
    for start, rows in ((3, [[3, 3], [3, 3]]), ([0, 14], [[0, 0], [14, 14]])):
        kd = dev(kc)
        vc.vitcop_cache_append(kd, None, dev(k), None, start=start)
        assert np.array_equal(host_bits(kd), np.stack(appended(kc, k, rows, None, None)))
        vd = dev(kc)
        vc.vitcop_cache_append(None, vd, None, dev(k), start=start)
        assert torch.equal(vd, kd)


def test_a_graph_goes_by_the_arrays(vc):
    B, T, Hq, Hkv, d, capacity = 2, 3, 4, 2, 64, 12
    rng = np.random.default_rng(8)
    q, k, v = (dev(bits(rng, (B, T, h, d))) for h in (Hq, Hkv, Hkv))
    pos, starts, counts, idx = ints(np.zeros((2, B, T))), ints([0, 0]), ints([0, 0]), ints(np.zeros((B, 2)))
    lstarts = ints(np.zeros((1, B)))

    def calls(kc, vcache, out):
        vc.vitcop_rope_axes(q, k, pos, (16, 16), v=v, cache=vc.Cache(kc, vcache), start_samples=starts, n_samples=counts, out=out)
        vc.vitcop_cache_append([kc], [vcache], k[None], v[None], start_samples=lstarts, idx=idx, n_samples=counts)

    state = [marked((B, capacity, Hkv, d)), marked((B, capacity, Hkv, d)), marked((B, T, Hq, d))]
    calls(*state)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(*state)
    for i in range(3):
        pos.copy_(torch.from_numpy(rng.integers(0, 100, (2, B, T)).astype(np.int32)))
        starts.copy_(torch.tensor([i, 5 - i], dtype=torch.int32))
        counts.copy_(torch.tensor([3 - i, 2], dtype=torch.int32))
        idx.copy_(torch.tensor([[i, 2], [0, 1]], dtype=torch.int32))
        lstarts.copy_(torch.tensor([[8, 9]], dtype=torch.int32))
        for t in state:
            t.copy_(marked(t.shape))
        g.replay()
        fresh = [marked(t.shape) for t in state]
        calls(*fresh)
        torch.cuda.synchronize()
        for a, b in zip(state, fresh):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert host_f64(state[2]).shape == (B, T, Hq, d)


def test_refusals_of_the_binding(vc):
    B, T, H, d = 2, 3, 2, 64
    q, k, v = (torch.zeros((B, T, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    pos = ints(np.zeros((2, B, T)))
    cache = vc.Cache(*[torch.zeros((B, 5, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    good = dict(q=q, k=k, positions=pos, sections=(16, 16))
    for bad in (dict(sections=(16, 15)), dict(sections=()), dict(sections=(16, 16, 0)), dict(sections=(2 ** 33, 32)),
                dict(sections=(-1, 33)), dict(positions=pos.long()), dict(positions=pos[:, :1]), dict(positions=pos.cpu()),
                dict(theta=1.0), dict(theta=float("inf")), dict(q=None, k=None), dict(v=v), dict(start=1), dict(k=k[:, :2]),
                dict(q=q.float()), dict(out=k[:, :2]), dict(k_out=q.half()), dict(q=None, out=q), dict(k=None, k_out=k),
                dict(cache=cache, k_out=k), dict(cache=cache, start=3), dict(cache=cache, start=-1), dict(k=None, cache=cache),
                dict(cache=cache, start_samples=pos[0, 0]), dict(n_samples=pos[0]), dict(k=k[..., :32], cache=cache),
                dict(q=q[..., 1:], k=None), dict(q=q[:, :1].expand(B, T, H, d), out=q[:, :1].expand(B, T, H, d))):
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_rope_axes(**dict(good, **bad))
    kc, idx, at = k[None], pos[0, :, :2].contiguous(), pos[:1, :, 0].contiguous()
    good = dict(k_caches=[cache.k], v_caches=[cache.v], k=kc, v=kc, start=0)
    for bad in (dict(k=None, v=None), dict(start=None), dict(start=3), dict(start=[0, 0]), dict(start=-1), dict(start=2 ** 31),
                dict(start_samples=at), dict(k=k), dict(k=kc.float()), dict(k_caches=None), dict(k_caches=[]),
                dict(k_caches=[cache.k] * 2), dict(k_caches=[cache.k[:, :4].contiguous()]), dict(k_caches=cache.k),
                dict(idx=idx.long()), dict(idx=idx[0]), dict(idx=idx[:1]), dict(n_samples=at), dict(start=None, start_samples=idx),
                dict(v=kc[:, :, :2]), dict(k=kc.cpu()), dict(k=torch.cat([kc, kc], 3)[:, :, :, ::2])):
        with pytest.raises((ValueError, vc.VitcopError)):
            vc.vitcop_cache_append(**dict(good, **bad))
    vc.vitcop_cache_append(**good)
