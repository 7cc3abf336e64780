"""The calls in 4 bits as a program uses them: a decoding layer with every stage against the oracle, and captured graphs whose
inputs change and whose outputs are cleared between replays."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from oracle import decoder_oracle as Dc
from oracle import mx4_oracle as X
from oracle import vitcop_oracle as O
from gpu_util import dev, host_bits
from test_gpu_mx4 import EPS, decode_layer, i32, layer_setup, vc          # noqa: F401  (vc: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hq,Hkv,d", [(3, 4, 2, 64), (1, 2, 2, 128), (20, 6, 1, 64)])
def test_norms_queries_and_keys_of_a_decoding_layer(vc, B, Hq, Hkv, d):          # noqa: F811
    D, F, N = 256, 384, 90
    c, w, wd, w4 = layer_setup(vc, B, D, Hq, Hkv, d, F, N, N)
    cache = vc.CacheMx4.empty(B, N, Hkv, d)
    rows = [I.normal_bf16(1700, i, (B, N, Hkv, d)) for i in range(2)]
    vc.vitcop_cache_mx4_write(cache, dev(rows[0]), dev(rows[1]))
    cached = [(17 * b) % (N - 1) for b in range(B)]
    positions = [[100 + b] for b in range(B)]
    h = I.normal_bf16(1701, 0, (B, D))
    s = decode_layer(vc, dev(h), w4, wd["ln1"], wd["ln2"], cache, i32(cached), N, i32(positions), Hq, Hkv, d)
    g = {k: host_bits(t) for k, t in s.items()}
    # half a step of the output; before it a sum of D squares, a square root and two products
    for name, x, ln in (("a", h, "ln1"), ("b", g["h1"], "ln2")):
        ref = Dc.rmsnorm(x, w[ln], 1e-5)
        assert (np.abs(O.bf16_to_f64(g[name]) - ref) <= (2.0 ** -8 + (D + 8) * EPS) * np.abs(ref)).all(), name
    # a projected value is off by half a step and what its sum carries, a turned one by that of both of its pair, by half a step
    # of itself and by the angle: up to 123 radians of frequencies good to 7.4e-7 (the exponent 13.3 in 32 bits, its power of two
    # and the product)
    for name, heads in (("q", Hq), ("k", Hkv)):
        xv, wv = O.bf16_to_f64(g["a"]), X.round_trip(w["w" + name])
        p, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
        p, off = (t.reshape(B, 1, heads, d) for t in (p, 2.0 ** -8 * np.abs(p) + (D + 4) * EPS * size))
        half = d // 2
        angle = np.asarray(positions, dtype=np.float64)[:, :, None, None] * 10000.0 ** (-np.arange(half) * 2.0 / d)
        cs, sn = np.cos(angle), np.sin(angle)
        lo, hi = p[..., :half], p[..., half:]
        ref = np.concatenate([lo * cs - hi * sn, hi * cs + lo * sn], -1)
        off_lo, off_hi = off[..., :half], off[..., half:]
        before = np.concatenate([off_lo * np.abs(cs) + off_hi * np.abs(sn), off_hi * np.abs(cs) + off_lo * np.abs(sn)], -1)
        pair = np.concatenate([np.hypot(lo, hi)] * 2, -1)
        bound = 2.0 ** -8 * np.abs(ref) + 1.01 * before + 1e-4 * pair
        assert (np.abs(O.bf16_to_f64(g[name]) - ref) <= bound).all(), name
    # the new row alone changed, and attention saw it
    for side, (x, new) in enumerate(((rows[0], "k"), (rows[1], "v"))):
        want = X.round_trip(x).transpose(0, 2, 1, 3).copy()
        for b in range(B):
            want[b, :, cached[b]] = X.round_trip(g[new])[b, 0]
        codes, scales = ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))[side]
        got = X.values(codes.cpu().numpy(), scales.cpu().numpy())
        assert np.array_equal(got, want)
        rows[side] = got
    ref, _, spread, size = X.decode_attention(g["q"][:, 0], rows[0], rows[1], [n + 1 for n in cached])
    p_off = (d + 4) * EPS * size + 2.0 ** -20 + N * EPS
    assert (np.abs(O.bf16_to_f64(g["o"]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2 * p_off[..., None] * spread).all()


def graph_inputs(B, N, Hq, Hkv, d, shapes, sets):
    return [dict(q=dev(I.normal_bf16(1800 + s, 0, (B, Hq, d))), k=dev(I.normal_bf16(1800 + s, 1, (B, N, Hkv, d))),
                 v=dev(I.normal_bf16(1800 + s, 2, (B, N, Hkv, d))),
                 xs=[dev(I.normal_bf16(1800 + s, 3 + j, (m, k))) for j, (m, _, k) in enumerate(shapes)]) for s in range(sets)]


@pytest.mark.parametrize("shared", [False, True])
def test_graphs_with_workspaces_on_changing_inputs(vc, shared):          # noqa: F811
    """A cache written, sliced attention over it, a sliced projection and one by way of bf16, in two graphs.  Before every turn
    both graphs' inputs get other values and all their outputs NaN, so that nothing left from the turn before is right: with
    workspaces of their own the graphs run in turn and at once on two streams, eager calls between; with one workspace that both
    were given, in turn."""
    B, N, Hq, Hkv, d, shapes = 3, 2000, 8, 2, 128, [(316, 640, 4448), (700, 4096, 256)]
    inputs = graph_inputs(B, N, Hq, Hkv, d, shapes, 3)
    matrices = [vc.vitcop_mx4_quantize(dev(I.normal_bf16(1850, j, (n, k), std=0.02))) for j, (_, n, k) in enumerate(shapes)]
    need = [vc.lib.vitcop_decode_attn_mx4_workspace_bytes(B, N, Hq, Hkv, d)]
    need += [vc.lib.vitcop_project_mx4_workspace_bytes(*s) for s in shapes]
    assert all(need) and need[2] >= 2 * shapes[1][1] * shapes[1][2]
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda") if shared else None

    def calls(x, cache, out):
        vc.vitcop_cache_mx4_write(cache, x["k"], x["v"])
        vc.vitcop_decode_attn_mx4(x["q"], cache, N, out=out[0], ws=ws)
        for a, m, y in zip(x["xs"], matrices, out[1:]):
            vc.vitcop_project_mx4(a, *m, out=y, ws=ws)

    def outputs():
        return [(torch.empty_like(inputs[0]["q"]), torch.empty((B, Hq), device="cuda"))] + \
               [torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for m, n, _ in shapes]

    flat = lambda out: [*out[0], *out[1:]]          # noqa: E731
    eager_cache = vc.CacheMx4.empty(B, N, Hkv, d)
    want = []
    for x in inputs:
        out = outputs()
        calls(x, eager_cache, out)
        want.append([t.clone() for t in flat(out)])
    assert not any(torch.equal(a, b) for a, b in zip(want[0], want[1]))
    graphs = []
    for g in range(2):
        x = {n: t.clone() if n != "xs" else [y.clone() for y in t] for n, t in inputs[g].items()}
        entry = (torch.cuda.CUDAGraph(), x, vc.CacheMx4.empty(B, N, Hkv, d), outputs(), torch.cuda.Stream())
        calls(entry[1], entry[2], entry[3])
        torch.cuda.synchronize()
        with torch.cuda.graph(entry[0]):
            calls(entry[1], entry[2], entry[3])
        graphs.append(entry)
    eager = outputs()
    for turn in range(6):
        for g, (_, x, _, out, _) in enumerate(graphs):
            new = inputs[(turn + g) % 3]
            for name in ("q", "k", "v"):
                x[name].copy_(new[name])
            for a, b in zip(x["xs"], new["xs"]):
                a.copy_(b)
            for t in flat(out):
                t.fill_(float("nan"))
        for t in flat(eager):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, _, _, _, stream in graphs:
            if shared or turn % 2 == 0:
                graph.replay()
            else:
                with torch.cuda.stream(stream):
                    graph.replay()
        calls(inputs[(turn + 2) % 3], eager_cache, eager)
        torch.cuda.synchronize()
        for g, (_, _, _, out, _) in enumerate(graphs):
            assert all(torch.equal(a, b) for a, b in zip(flat(out), want[(turn + g) % 3])), (turn, g)
        assert all(torch.equal(a, b) for a, b in zip(flat(eager), want[(turn + 2) % 3])), turn
