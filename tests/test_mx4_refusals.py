"""What the calls on 4-bit caches and weights refuse, on the host and before any HIP call: nothing here needs a GPU."""
import ctypes as C

import pytest
import torch

from paper_2601_17818_amd import binding as vc

lib = vc.lib
A = 0x1000              # a fake, aligned, non-null device pointer (never dereferenced)
EINVAL, EUNSUPPORTED, EWORKSPACE, OK = vc.VITCOP_EINVAL, vc.VITCOP_EUNSUPPORTED, vc.VITCOP_EWORKSPACE, vc.VITCOP_OK


def test_struct_layout():
    assert C.sizeof(vc.CacheMx4T) == 4 * 4 + 4 * 8


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), EINVAL), (dict(K=0), EINVAL), (dict(K=48, stride=48), EUNSUPPORTED), (dict(stride=56), EINVAL),
    (dict(stride=68), EINVAL), (dict(a=None), EINVAL), (dict(b=None), EINVAL), (dict(c=None), EINVAL), (dict(a=A + 8), EINVAL),
    (dict(b=A + 4), EINVAL), (dict(c=A + 1), EINVAL), (dict(M=1 << 28), EUNSUPPORTED), (dict(M=0, a=None, b=None, c=None), OK)])
def test_rows(change, code):
    p = dict(dict(M=4, K=64, stride=64, a=A, b=A, c=A), **change)
    assert lib.vitcop_mx4_quantize(p["a"], p["stride"], p["M"], p["K"], p["b"], p["c"], None) == code
    assert lib.vitcop_mx4_dequantize(p["b"], p["c"], p["M"], p["K"], p["a"], p["stride"], None) == code


def cache(B=2, capacity=64, Hkv=2, d=128, kc=A, ks=A, v=A, vs=A):
    return vc.CacheMx4T(B, capacity, Hkv, d, kc, ks, v, vs)


CACHES = [(dict(B=-1), EINVAL), (dict(capacity=-1), EINVAL), (dict(Hkv=0), EINVAL), (dict(d=96), EUNSUPPORTED),
          (dict(B=65536), EUNSUPPORTED), (dict(Hkv=65536), EUNSUPPORTED), (dict(capacity=1 << 24), EUNSUPPORTED),
          (dict(kc=None), EINVAL), (dict(vs=None), EINVAL), (dict(ks=A + 2), EINVAL), (dict(v=A + 8), EINVAL)]


@pytest.mark.parametrize("change,code", CACHES)
def test_descriptor(change, code):
    c = C.byref(cache(**change))
    assert lib.vitcop_cache_mx4_write(c, A, A, 256, 512, 2, 0, None, None, None) == code
    assert lib.vitcop_cache_mx4_read(c, A, A, 2, 0, None, None) == code
    assert lib.vitcop_decode_attn_mx4(A, c, A, None, 8, None, 4, 0.0, A, 1 << 30, None) == code


def test_a_null_descriptor():
    assert lib.vitcop_cache_mx4_write(None, A, A, 256, 512, 2, 0, None, None, None) == EINVAL
    assert lib.vitcop_cache_mx4_read(None, A, A, 2, 0, None, None) == EINVAL
    assert lib.vitcop_decode_attn_mx4(A, None, A, None, 8, None, 4, 0.0, A, 1 << 30, None) == EINVAL


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), EINVAL), (dict(start=-1), EINVAL), (dict(start=63), EINVAL), (dict(T=65), EINVAL), (dict(k=None, v=None), EINVAL),
    (dict(start=2147483647), EINVAL), (dict(k=A + 4), EINVAL), (dict(v=A + 8), EINVAL), (dict(T=0, k=None, v=None), OK)])
def test_rows_of_a_cache(change, code):
    p = dict(dict(k=A, v=A, T=2, start=0), **change)
    c = C.byref(cache())
    assert lib.vitcop_cache_mx4_write(c, p["k"], p["v"], 256, 512, p["T"], p["start"], None, None, None) == code
    assert lib.vitcop_cache_mx4_read(c, p["k"], p["v"], p["T"], p["start"], None, None) == code


def test_strides_and_sizes_of_a_cache():
    w = lib.vitcop_cache_mx4_write
    c = C.byref(cache())
    assert w(c, A, A, 252, 512, 2, 0, None, None, None) == EINVAL
    assert w(c, A, A, 256, 516, 2, 0, None, None, None) == EINVAL
    assert w(c, A, A, -256, 512, 2, 0, None, None, None) == EINVAL
    big = C.byref(cache(B=65535, Hkv=2048, capacity=1))
    assert w(big, A, A, 256, 512, 1, 0, None, None, None) == EUNSUPPORTED
    assert lib.vitcop_cache_mx4_read(big, A, A, 1, 0, None, None) == EUNSUPPORTED
    empty = C.byref(cache(B=0, kc=None, ks=None, v=None, vs=None))
    assert w(empty, None, None, 256, 512, 2, 0, None, None, None) == OK
    assert lib.vitcop_cache_mx4_read(empty, None, None, 2, 0, None, None) == OK
    assert lib.vitcop_decode_attn_mx4(None, empty, None, None, 8, None, 4, 0.0, None, 0, None) == OK
    # nothing to write to: rows that all lie outside
    assert w(C.byref(cache(capacity=0)), A, A, 256, 512, 2, 0, A, None, None) == OK
    # only one side is asked for: the other may be missing
    assert w(C.byref(cache(v=None, vs=None)), A, None, 256, 512, 65, 0, None, None, None) == EINVAL     # (the rows are checked)
    assert "rows" in vc.vitcop_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(N=4097), EINVAL), (dict(N=-1), EINVAL), (dict(Hq=3), EINVAL), (dict(Hq=0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
    (dict(q=A + 8), EINVAL), (dict(out=A + 2), EINVAL), (dict(ws=A + 4), EINVAL), (dict(ws=None), EWORKSPACE),
    (dict(nb=16), EWORKSPACE), (dict(Hq=1 << 24), EUNSUPPORTED)])
def test_attention(change, code):
    p = dict(dict(q=A, out=A, N=4096, Hq=4, scale=0.0, ws=A, nb=1 << 30), **change)
    c = C.byref(cache(capacity=4096))
    assert lib.vitcop_decode_attn_mx4(p["q"], c, p["out"], None, p["N"], None, p["Hq"], p["scale"], p["ws"], p["nb"], None) == code


def test_attention_workspace():
    f = lib.vitcop_decode_attn_mx4_workspace_bytes
    assert f(2, 4096, 4, 2, 128) > 0 and f(2, 64, 4, 2, 128) == 0 and f(2, 0, 4, 2, 128) == 0
    assert f(2, 64, 4, 3, 128) == 0 and f(2, 64, 4, 2, 32) == 0 and f(-1, 64, 4, 2, 128) == 0


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), EINVAL), (dict(N=-16), EINVAL), (dict(K=0), EINVAL), (dict(K=48, xs=48), EUNSUPPORTED), (dict(N=24), EUNSUPPORTED),
    (dict(xs=56), EINVAL), (dict(xs=68), EINVAL), (dict(ys=24), EINVAL), (dict(ys=36), EINVAL), (dict(rs=24), EINVAL),
    (dict(M=(1 << 20) + 1), EUNSUPPORTED), (dict(M=1 << 20, xs=1024), EUNSUPPORTED), (dict(N=1 << 26, ys=1 << 26, rs=1 << 26),
                                                                                        EUNSUPPORTED),
    (dict(x=None), EINVAL), (dict(c=None), EINVAL), (dict(s=None), EINVAL), (dict(y=None), EINVAL), (dict(x=A + 8), EINVAL),
    (dict(c=A + 4), EINVAL), (dict(s=A + 1), EINVAL), (dict(y=A + 8), EINVAL), (dict(r=A + 8), EINVAL), (dict(ws=A + 8), EINVAL),
    (dict(M=0, x=None), OK), (dict(N=0, ys=0, rs=0, y=None), OK)])
def test_projection(change, code):
    p = dict(dict(x=A, xs=64, c=A, s=A, y=A, ys=32, r=A, rs=32, M=4, N=32, K=64, ws=None), **change)
    assert lib.vitcop_project_mx4(p["x"], p["xs"], p["c"], p["s"], p["y"], p["ys"], p["r"], p["rs"], p["M"], p["N"], p["K"],
                                  p["ws"], 0, None) == code


def test_the_binding_refuses_host_tensors():
    x, u8 = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 32, dtype=torch.uint8)
    for call in (lambda: vc.vitcop_mx4_quantize(x), lambda: vc.vitcop_mx4_dequantize(u8, u8[:, :2]),
                 lambda: vc.vitcop_project_mx4(x, u8, u8[:, :2]), lambda: vc.CacheMx4.empty(1, 8, 2, 64, device="cpu")):
        with pytest.raises(ValueError, match="CUDA"):
            call()
