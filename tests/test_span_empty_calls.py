"""Calls on prompts, tokens and drafts over a bf16 cache without a sample or a token, of views of fused rows.  They return before
any HIP call, so the binding is given tensors of the host."""
import pytest
import torch

from paper_2601_17818_amd import binding as vc

HQ, HKV, D = 8, 2, 64
EMPTY = [(2, 0), (0, 3), (0, 0), (1, 0), (0, 1)]


@pytest.fixture(autouse=True)
def host(monkeypatch):
    monkeypatch.setattr(vc, "_here", lambda t, name: t.get_device())
    monkeypatch.setattr(vc, "_stream_of", lambda device: 0)


def rows(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def fused(B, T):
    """q, k, v of rows that hold more than they, samples further apart than their tokens."""
    wide = rows(B, T + 2, HQ + 2 * HKV + 1, D)[:, :T]
    return wide[:, :, :HQ], wide[:, :, HQ:HQ + HKV], wide[:, :, HQ + HKV:HQ + 2 * HKV]


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("B,T", EMPTY)
def test_rope_axes(B, T):
    q, k, v = fused(B, T)
    pos = ints(2, B, T)
    out, k_out = vc.vitcop_rope_axes(q, k, pos, (16, 16))
    assert out.shape == q.shape and k_out.shape == k.shape
    given = vc.vitcop_rope_axes(q, k, pos, (16, 16), out=out, k_out=k_out)
    assert given[0] is out and given[1] is k_out
    assert vc.vitcop_rope_axes(q, k, pos, (16, 16), out=q, k_out=k) == (q, k)
    assert vc.vitcop_rope_axes(None, k, pos, (16, 16))[1].shape == k.shape
    cache = vc.Cache(rows(B, 5, HKV, D), rows(B, 5, HKV, D))
    out, none = vc.vitcop_rope_axes(q, k, pos, (16, 16), v=v, cache=cache, start_samples=ints(B), n_samples=ints(B))
    assert out.shape == q.shape and none is None
    with pytest.raises(ValueError):
        vc.vitcop_rope_axes(q, k, pos, (16, 16), out=rows(B, T, HQ + 1, D))
    with pytest.raises(ValueError):
        vc.vitcop_rope_axes(q, k, pos, (16, 16), k_out=rows(B, T, HKV, D + 16))


def test_rope_axes_without_heads():
    wide = rows(2, 3, 4, D)
    out, k_out = vc.vitcop_rope_axes(wide[:, :, :0], wide[:, :, 4:], ints(2, 2, 3), (16, 16))
    assert out.shape == k_out.shape == (2, 3, 0, D)


@pytest.mark.parametrize("B,T", EMPTY)
def test_attention(B, T):
    q, k, v = fused(B, T)
    cache = vc.Cache(rows(B, 5, HKV, D), rows(B, 5, HKV, D))
    masks = torch.zeros((B, T), dtype=torch.int64)
    for out, lse in (vc.vitcop_window_attn(q, cache, 1, 3, 1, ints(B), ints(B)), vc.vitcop_tree_attn(q, k, v, masks, cache, 1)):
        assert out.shape == (B, T, HQ, D) and lse.shape == (B, HQ, T)


@pytest.mark.parametrize("B,T", EMPTY)
@pytest.mark.parametrize("stacked", [True, False])
def test_cache_append(B, T, stacked):
    L = 3
    caches = rows(L, B, 5, HKV, D)
    caches = caches if stacked else list(caches)
    wide = rows(L, B, T + 2, 2 * HKV, D)[:, :, :T]
    vc.vitcop_cache_append(caches, caches, wide[:, :, :, :HKV], wide[:, :, :, HKV:], start_samples=ints(L, B))


@pytest.mark.parametrize("stacked", [True, False])
def test_cache_append_of_paths_through_no_token(stacked):
    """Every source is outside of no rows: nothing is written."""
    caches = rows(3, 2, 5, HKV, D)
    caches = caches if stacked else list(caches)
    wide = rows(3, 2, 0, 2 * HKV, D)
    vc.vitcop_cache_append(caches, caches, wide[:, :, :, :HKV], wide[:, :, :, HKV:], start=1, idx=ints(2, 4))
    vc.vitcop_cache_append(caches, None, wide[:, :, :, :HKV], None, start_samples=ints(3, 2), idx=ints(2, 4))
