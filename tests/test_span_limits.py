"""The limits of the calls over a bf16 cache, at the last size that is taken and the first that is not (nothing here needs a GPU:
what is taken is refused for a null pointer afterwards)."""
import ctypes as C

import pytest

from test_span_refusals import EINVAL, EUNSUPPORTED, append, cache, rope, tree, window


def of(**sizes):
    return C.byref(cache(**sizes))


@pytest.mark.parametrize("last,code", [(1 << 30, EINVAL), ((1 << 30) + 1, EUNSUPPORTED)])
def test_rows(last, code):
    assert window(of(B=1, capacity=last, Hkv=1), T=1, start=last - 1, Hq=1, q=None) == code
    assert tree(of(B=1, capacity=1 << 30, Hkv=1), T=1, start=last - 1, Hq=1, q=None) == code


@pytest.mark.parametrize("Hkv,code", [(2047, EINVAL), (2048, EUNSUPPORTED)])
def test_samples_times_heads(Hkv, code):
    for call in (window, tree):
        assert call(of(B=4096, capacity=9, Hkv=Hkv), T=1, start=0, Hq=Hkv, q=None) == code


@pytest.mark.parametrize("T,Hq,code", [(1, (1 << 28) - 1, EINVAL), (1, 1 << 28, EUNSUPPORTED), (63, 4260880, EINVAL),
                                       (64, 1 << 22, EUNSUPPORTED)])
def test_query_heads(T, Hq, code):
    for call in (window, tree):
        assert call(of(B=1, capacity=99, Hkv=1), T=T, start=9, Hq=Hq, q=None) == code


@pytest.mark.parametrize("row,batch,code", [((1 << 31) - 8, (1 << 46) - 8, EINVAL), (1 << 31, 2048, EUNSUPPORTED),
                                            (512, 1 << 46, EUNSUPPORTED)])
def test_strides(row, batch, code):
    assert window(row=row, batch=batch, q=None) == tree(row=row, batch=batch, q=None) == code
    assert rope(q_row=row, q_batch=batch, positions=None if code == EINVAL else 16) == code
    assert append(kr=row, kb=batch, k_cache=(C.c_void_p * 2)(None, None)) == code


@pytest.mark.parametrize("row,code", [((1 << 24) - 8, EINVAL), (1 << 24, EUNSUPPORTED)])
def test_rows_of_drafts(row, code):
    assert tree(k_row=row, q=None) == tree(v_row=row, q=None) == code
