"""What the calls on prompts, tokens and drafts over a bf16 cache refuse, on the host and before any HIP call: nothing here
needs a GPU."""
import ctypes as C

import pytest

from paper_2601_17818_amd import binding as vc

lib = vc.lib
A = 0x1000              # a fake, aligned, non-null device pointer (never dereferenced)
EINVAL, EUNSUPPORTED, EWORKSPACE, OK = vc.VITCOP_EINVAL, vc.VITCOP_EUNSUPPORTED, vc.VITCOP_EWORKSPACE, vc.VITCOP_OK
BIG = 2147483647
Sections = C.c_int * vc.VITCOP_MAX_AXES


class CacheT(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("B", "capacity", "Hkv", "d")] + [("k", C.c_void_p), ("v", C.c_void_p)])


class RopeAxesT(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("B", "T", "Hq", "Hkv", "d", "n_axes", "interleaved")] +
                [("sections", Sections), ("theta", C.c_float), ("capacity", C.c_int), ("start", C.c_int)] +
                [(n, C.c_void_p) for n in ("positions", "q", "k", "v")] +
                [(n, C.c_int64) for n in ("q_row_stride", "q_batch_stride", "k_row_stride", "k_batch_stride",
                                           "v_row_stride", "v_batch_stride")] +
                [(n, C.c_void_p) for n in ("q_out", "k_out", "v_out", "start_samples", "n_samples")])


class CacheAppendT(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("n_layers", "B", "capacity", "Hkv", "d", "T", "rows")] +
                [("k_cache", C.POINTER(C.c_void_p)), ("v_cache", C.POINTER(C.c_void_p)), ("cache_layer_stride", C.c_int64),
                 ("k", C.c_void_p), ("v", C.c_void_p)] +
                [(n, C.c_int64) for n in ("k_layer_stride", "k_batch_stride", "k_row_stride",
                                           "v_layer_stride", "v_batch_stride", "v_row_stride")] +
                [("start", C.POINTER(C.c_int))] + [(n, C.c_void_p) for n in ("start_samples", "idx", "n_samples")])


def test_struct_layouts():
    assert vc._CACHE.size == 32 and vc._ROPE_AXES.size == 176 and vc._CACHE_APPEND.size == 152
    assert C.sizeof(CacheT) == 32 and C.sizeof(RopeAxesT) == 176 and C.sizeof(CacheAppendT) == 152


def test_packed_descriptors():
    """The binding's bytes are the structures'."""
    for packed, kind in ((vc._CACHE, CacheT), (vc._ROPE_AXES, RopeAxesT), (vc._CACHE_APPEND, CacheAppendT)):
        s = kind()
        n, flat = 1, []
        for name, field in kind._fields_:
            if field is Sections:
                s.sections = Sections(*range(n, n + 4))
                flat += range(n, n + 4)
                n += 4
                continue
            setattr(s, name, C.cast(n * 16, field) if issubclass(field, C._Pointer) else n * 16)
            flat.append(n * 16)
            n += 1
        assert packed.pack(*flat) == bytes(s)


def cache(B=2, capacity=64, Hkv=2, d=128, k=A, v=A):
    return CacheT(B, capacity, Hkv, d, k, v)


CACHES = [(dict(B=-1), EINVAL), (dict(capacity=-1), EINVAL), (dict(Hkv=0), EINVAL), (dict(d=96), EUNSUPPORTED),
          (dict(B=65536), EUNSUPPORTED), (dict(Hkv=65536), EUNSUPPORTED), (dict(capacity=(1 << 30) + 1), EUNSUPPORTED),
          (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=A + 8), EINVAL), (dict(v=A + 2), EINVAL), (dict(B=0), OK)]


def window(c=None, **change):
    p = dict(dict(q=A, row=512, batch=2048, out=A, lse=None, T=4, start=8, Hq=4, window=0, sinks=0, scale=0.0, ws=A, n=1 << 40),
             **change)
    return lib.vitcop_window_attn(p["q"], p["row"], p["batch"], c if c is not None else C.byref(cache()), p["out"], p["lse"], p["T"],
                                  p["start"], None, None, p["Hq"], p["window"], p["sinks"], p["scale"], p["ws"], p["n"], None)


def tree(c=None, **change):
    p = dict(dict(q=A, row=512, batch=2048, k=A, k_row=256, k_batch=1024, v=A, v_row=256, v_batch=1024, tree=A, t_batch=4, out=A,
                  T=4, start=8, Hq=4, scale=0.0, ws=A, n=1 << 40), **change)
    return lib.vitcop_tree_attn(p["q"], p["row"], p["batch"], c if c is not None else C.byref(cache()), p["k"], p["k_row"],
                                p["k_batch"], p["v"], p["v_row"], p["v_batch"], p["tree"], p["t_batch"], p["out"], None, p["T"],
                                p["start"], None, None, p["Hq"], p["scale"], p["ws"], p["n"], None)


@pytest.mark.parametrize("change,code", CACHES)
def test_descriptor(change, code):
    assert window(C.byref(cache(**change))) == code and tree(C.byref(cache(**change))) == code


def test_null_descriptors():
    null = C.POINTER(CacheT)()
    assert window(null) == EINVAL and tree(null) == EINVAL
    assert lib.vitcop_rope_axes(None, None) == EINVAL and lib.vitcop_cache_append(None, None) == EINVAL


BOTH = [(dict(T=-1), EINVAL), (dict(start=-1), EINVAL), (dict(Hq=3), EINVAL), (dict(Hq=0), EINVAL), (dict(row=-8), EINVAL),
        (dict(row=516), EINVAL), (dict(batch=2052), EINVAL), (dict(batch=-8), EINVAL), (dict(row=1 << 31), EUNSUPPORTED),
        (dict(batch=1 << 46), EUNSUPPORTED), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q=A + 8), EINVAL),
        (dict(out=A + 4), EINVAL), (dict(ws=A + 8), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL),
        (dict(scale=float("inf")), EINVAL), (dict(start=65), EINVAL), (dict(start=BIG), EUNSUPPORTED), (dict(Hq=1 << 27), EUNSUPPORTED),
        (dict(T=0, q=None, out=None), OK)]


@pytest.mark.parametrize("change,code", BOTH)
def test_attention(change, code):
    assert window(**change) == code and tree(**change) == code


@pytest.mark.parametrize("change,code", [(dict(start=61), EINVAL), (dict(T=57), EINVAL), (dict(window=-1), EINVAL),
                                         (dict(sinks=-1), EINVAL), (dict(T=BIG, start=1), EUNSUPPORTED)])
def test_windows(change, code):
    assert window(**change) == code


@pytest.mark.parametrize("change,code", [
    (dict(T=65), EUNSUPPORTED), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(tree=None), EINVAL), (dict(tree=A + 4), EINVAL),
    (dict(k=A + 8), EINVAL), (dict(v=A + 8), EINVAL), (dict(k_row=248), EINVAL), (dict(v_row=128), EINVAL), (dict(v_row=260), EINVAL),
    (dict(k_batch=-1024), EINVAL), (dict(k_row=1 << 24), EUNSUPPORTED), (dict(v_row=1 << 24), EUNSUPPORTED), (dict(t_batch=3), EINVAL), (dict(t_batch=-4), EINVAL),
    (dict(t_batch=1 << 31), EUNSUPPORTED)])
def test_trees(change, code):
    assert tree(**change) == code


def test_more_query_rows_than_a_grid_has_blocks_for():
    """65535 blocks of 32 rows, where a cache of 4 GiB and more leaves the kernel of many rows out."""
    c = C.byref(cache(B=1, capacity=1 << 22, Hkv=32))
    row = 32 * 128
    assert window(c, T=32 * 65535 + 1, start=0, Hq=32, row=row) == EUNSUPPORTED
    assert b"query rows" in lib.vitcop_last_error()


def test_workspaces():
    c = C.byref(cache(B=1, capacity=5000, Hkv=1))
    for need, call in ((lib.vitcop_window_attn_workspace_bytes(1, 1, 4000, 1, 1, 128, 0, 0), window),
                       (lib.vitcop_tree_attn_workspace_bytes(1, 1, 4000, 1, 1, 128), tree)):
        assert need > 0
        assert call(c, T=1, start=4000, Hq=1, ws=None, n=0) == EWORKSPACE
        assert call(c, T=1, start=4000, Hq=1, n=need - 1) == EWORKSPACE
    for sizes in ((-1, 1, 9, 4, 2, 128), (1, 1, 9, 3, 2, 128), (1, 1, 9, 4, 2, 96), (1, -1, 9, 4, 2, 64), (0, 1, 4000, 4, 2, 64),
                  (1, 1, BIG, 1, 1, 128), (65535, 1, 9, 65535, 65535, 64)):
        assert lib.vitcop_window_attn_workspace_bytes(*sizes, 0, 0) == lib.vitcop_tree_attn_workspace_bytes(*sizes) == 0
    assert lib.vitcop_window_attn_workspace_bytes(1, 1, 4000, 1, 1, 128, -1, 0) == 0
    assert lib.vitcop_window_attn_workspace_bytes(1, 1, 4000, 1, 1, 128, 0, -1) == 0
    assert lib.vitcop_tree_attn_workspace_bytes(1, 65, 4000, 1, 1, 128) == 0


def rope(**change):
    p = dict(dict(B=2, T=3, Hq=4, Hkv=2, d=64, n_axes=3, interleaved=0, sections=(8, 12, 12), theta=10000.0, capacity=16, start=5,
                  positions=A, q=A, k=A, v=A, q_row=512, q_batch=1536, k_row=512, k_batch=1536, v_row=512, v_batch=1536,
                  q_out=2 * A, k_out=3 * A, v_out=4 * A, start_samples=None, n_samples=None), **change)
    p["sections"] = (C.c_int * 4)(*p["sections"])
    return lib.vitcop_rope_axes(C.byref(RopeAxesT(*p.values())), None)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), EINVAL), (dict(T=-1), EINVAL), (dict(Hq=-1), EINVAL), (dict(Hkv=-1), EINVAL), (dict(d=0), EINVAL),
    (dict(d=72, sections=(36, 0, 0)), EUNSUPPORTED), (dict(d=272, sections=(136, 0, 0)), EUNSUPPORTED), (dict(n_axes=0), EINVAL),
    (dict(n_axes=5), EINVAL), (dict(sections=(8, 12, 11)), EINVAL), (dict(sections=(-8, 28, 12)), EINVAL),
    (dict(sections=(BIG, BIG, 34)), EINVAL), (dict(theta=1.0), EINVAL), (dict(theta=float("inf")), EINVAL),
    (dict(theta=float("nan")), EINVAL), (dict(capacity=-1), EINVAL), (dict(start=-1), EINVAL), (dict(start=14), EINVAL),
    (dict(start=BIG), EINVAL), (dict(positions=None), EINVAL), (dict(q_out=None), EINVAL), (dict(k_out=None), EINVAL),
    (dict(v_out=None), EINVAL), (dict(v_out=A), EINVAL), (dict(k_out=A), EINVAL), (dict(k_out=A, v=None), EINVAL),
    (dict(k_out=A, v=None, start=0, start_samples=A), EINVAL), (dict(q=A + 8), EINVAL), (dict(k=A + 8), EINVAL),
    (dict(v_out=A + 4), EINVAL), (dict(q_row=516), EINVAL), (dict(k_batch=-8), EINVAL), (dict(v_row=4), EINVAL),
    (dict(q_row=1 << 31), EUNSUPPORTED), (dict(k_batch=1 << 46), EUNSUPPORTED), (dict(Hq=65535), EUNSUPPORTED),
    (dict(T=BIG, start=0, capacity=BIG), EUNSUPPORTED), (dict(B=BIG), EUNSUPPORTED),
    (dict(q_out=A, q_row=248), EINVAL), (dict(q_out=A, q_batch=1024), EINVAL), (dict(q_out=A, q_batch=0), EINVAL),
    (dict(q_out=A, q_row=504, q_batch=256), EINVAL), (dict(k_out=A, v=None, start=0, k_row=120), EINVAL),
    (dict(B=0), OK), (dict(T=0), OK), (dict(q=None, k=None, v=None), OK), (dict(T=0, positions=None, q_out=None), OK)])
def test_rope_axes(change, code):
    assert rope(**change) == code


def append(**change):
    two, starts = (C.c_void_p * 2)(A, 2 * A), (C.c_int * 2)(0, 5)
    p = dict(dict(n_layers=2, B=2, capacity=9, Hkv=2, d=64, T=4, rows=4, k_cache=two, v_cache=two, cl=0, k=A, v=A, kl=1024, kb=512, kr=128,
                  vl=1024, vb=512, vr=128, start=starts, start_samples=None, idx=None, n_samples=None), **change)
    return lib.vitcop_cache_append(C.byref(CacheAppendT(*p.values())), None)


NULLS = C.POINTER(C.c_void_p)()


@pytest.mark.parametrize("change,code", [
    (dict(n_layers=-1), EINVAL), (dict(B=-1), EINVAL), (dict(capacity=-1), EINVAL), (dict(Hkv=0), EINVAL), (dict(d=0), EINVAL),
    (dict(T=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(rows=5), EINVAL), (dict(rows=5, idx=A), EINVAL), (dict(Hkv=1, d=12), EUNSUPPORTED),
    (dict(B=65536), EUNSUPPORTED), (dict(Hkv=1 << 16, d=1 << 16), EUNSUPPORTED), (dict(rows=1 << 24, T=1 << 24), EUNSUPPORTED),
    (dict(k=None, v=None), EINVAL), (dict(k_cache=NULLS), EINVAL), (dict(v_cache=NULLS), EINVAL),
    (dict(start=C.POINTER(C.c_int)()), EINVAL), (dict(k=A + 8), EINVAL), (dict(v=A + 8), EINVAL), (dict(kr=132), EINVAL),
    (dict(vb=-8), EINVAL), (dict(kl=-8), EINVAL), (dict(vl=4), EINVAL), (dict(kl=1 << 61), EINVAL), (dict(kb=1 << 46), EUNSUPPORTED),
    (dict(k_cache=(C.c_void_p * 2)(A, None)), EINVAL), (dict(v_cache=(C.c_void_p * 2)(A + 8, A)), EINVAL),
    (dict(start=(C.c_int * 2)(0, 6)), EINVAL), (dict(start=(C.c_int * 2)(-1, 0)), EINVAL), (dict(start=(C.c_int * 2)(BIG, 0)), EINVAL),
    (dict(cl=-8), EINVAL), (dict(cl=2 * 9 * 2 * 64 - 8), EINVAL), (dict(cl=2 * 9 * 2 * 64 + 4), EINVAL), (dict(cl=1 << 61), EINVAL),
    (dict(cl=1 << 40, k_cache=(C.c_void_p * 1)(A + 8)), EINVAL), (dict(cl=1 << 40, v_cache=(C.c_void_p * 1)(None)), EINVAL),
    (dict(cl=1 << 40, B=65535, capacity=BIG), EINVAL),
    (dict(n_layers=0), OK), (dict(B=0), OK), (dict(rows=0), OK)])
def test_cache_append(change, code):
    assert append(**change) == code
