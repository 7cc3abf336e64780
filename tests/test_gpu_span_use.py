"""A conversation's run of the calls on prompts, tokens and drafts, as a program makes it, against the same by single tokens."""
import numpy as np
import pytest
import torch

import vitcop_inputs as I
from gpu_util import dev, host_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,sections", [(8, 2, 128, (16, 24, 24)), (4, 4, 64, (8, 12, 12))])
def test_drafts_verified_and_taken_over(Hq, Hkv, d, sections):
    """Two layers, a right-padded batch: the prompt's rows turned into the caches and attended over; a tree of drafts turned,
    attended over, its accepted path appended; the next token.  Then the same conversation with the accepted tokens as part of
    the prompt: the caches are equal bit for bit, and the last token's results but for the sums' order."""
    from paper_2601_17818_amd import binding as vc
    L, B, P, T, capacity = 2, 3, 90, 12, 120
    rng = np.random.default_rng(1)

    def rows(n):
        return dev(I.f32_to_bf16_bits(rng.standard_normal((L, B, n, Hq + 2 * Hkv, d)).astype(np.float32)))

    def ints(x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

    lens = np.array([90, 41, 7])
    prompt, drafts, token = rows(P), rows(T), rows(1)
    pos = np.stack([np.arange(P) // 9, np.arange(P) // 3 % 3, np.arange(P) % 3])[:, None].repeat(B, 1)
    depth = np.array([0, 1, 1, 2, 2, 3, 3, 1, 2, 4, 5, 3])
    parent = [-1, 0, 0, 1, 2, 3, 4, 0, 7, 5, 9, 8]
    masks = []
    for t, p in enumerate(parent):
        masks.append((1 << t) | (masks[p] if p >= 0 else 0))
    path = np.array([[0, 1, 3, 5, 9], [0, 2, 4, 6, 6], [0, 7, 8, 11, 11]])
    n_path = np.array([5, 4, 2])
    draft_pos = np.broadcast_to(depth[None, None] + lens[None, :, None] + 100, (3, B, T))

    def split(x):
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]

    kc, vcache = (torch.zeros((L, B, capacity, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kept_k = torch.empty((L, B, T, Hkv, d), dtype=torch.bfloat16, device="cuda")
    tree = torch.tensor(masks, device="cuda")
    verified = []
    for layer in range(L):
        cache = vc.Cache(kc[layer], vcache[layer])
        q, k, v = split(prompt[layer])
        q, _ = vc.vitcop_rope_axes(q, k, ints(pos), sections, v=v, cache=cache, n_samples=ints(lens))
        vc.vitcop_window_attn(q, cache, 0, 30, 4, ints([0] * B), ints(lens))
        q, k, v = split(drafts[layer])
        q, _ = vc.vitcop_rope_axes(q, k, ints(draft_pos), sections, k_out=kept_k[layer])
        verified.append(vc.vitcop_tree_attn(q, kept_k[layer], v, tree, cache, P, start_samples=ints(lens)))
    vc.vitcop_cache_append(kc, vcache, kept_k, drafts[:, :, :, Hq + Hkv:], start_samples=ints(np.stack([lens] * L)),
                           idx=ints(path), n_samples=ints(n_path))
    now = lens + n_path
    last_pos = np.broadcast_to(now[None, :, None] + 100, (3, B, 1))

    def last(kc, vcache, layer):
        cache = vc.Cache(kc[layer], vcache[layer])
        q, k, v = split(token[layer])
        q, _ = vc.vitcop_rope_axes(q, k, ints(last_pos), sections, v=v, cache=cache, start_samples=ints(now))
        return vc.vitcop_window_attn(q, cache, int(now.max()), 0, 0, ints(now))

    # the same by single tokens
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vcache)
    for layer in range(L):
        for b in range(B):
            one = vc.Cache(kc2[layer, b:b + 1], vc2[layer, b:b + 1])
            q, k, v = split(prompt[layer, b:b + 1, :lens[b]])
            vc.vitcop_rope_axes(q, k, ints(pos[:, b:b + 1, :lens[b]]), sections, v=v, cache=one)
            for i in range(n_path[b]):
                t = path[b, i]
                q, k, v = split(drafts[layer, b:b + 1, t:t + 1])
                q, _ = vc.vitcop_rope_axes(q, k, ints(draft_pos[:, b:b + 1, t:t + 1]), sections, v=v, cache=one,
                                           start=int(lens[b]) + i)
                out, lse = vc.vitcop_window_attn(q, one, int(lens[b]) + i)
                got, glse = verified[layer][0][b, t], verified[layer][1][b, :, t]
                # two results of half a bf16 step each
                assert (got.float() - out[0, 0].float()).abs().max() <= 2.0 ** -7 * out.float().abs().max()
                assert (glse - lse[0, :, 0]).abs().max() < 1e-5
    assert np.array_equal(host_bits(kc), host_bits(kc2)) and np.array_equal(host_bits(vcache), host_bits(vc2))
    for layer in range(L):
        a, b = last(kc, vcache, layer), last(kc2, vc2, layer)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
