"""The limits of the calls on 4-bit caches and weights, at the last size that is taken and the first that is not (nothing here
needs a GPU: what is taken is refused for a null pointer afterwards)."""
import pytest

from paper_2601_17818_amd import binding as vc

lib = vc.lib
A = 0x1000              # a fake, aligned, non-null device pointer (never dereferenced)
EINVAL, EUNSUPPORTED, EWORKSPACE = vc.VITCOP_EINVAL, vc.VITCOP_EUNSUPPORTED, vc.VITCOP_EWORKSPACE
WRAPS = 1 << 45         # times 2^19 rows: 2^64, nothing in 64 bits


@pytest.mark.parametrize("M,xs,N,K,code", [
    (1 << 19, 64, 32, 64, EINVAL), ((1 << 19) + 1, 64, 32, 64, EUNSUPPORTED),
    (1 << 19, 2040, 32, 64, EINVAL), (1 << 19, 2048, 32, 64, EUNSUPPORTED),
    (1, (1 << 30) - 8, 32, 64, EINVAL), (1, 1 << 30, 32, 64, EUNSUPPORTED),
    (1 << 19, WRAPS, 32, 64, EUNSUPPORTED), (1 << 19, 5 * WRAPS, 32, 64, EUNSUPPORTED), (3, (1 << 63) - 8, 32, 64, EUNSUPPORTED),
    (4, 65536, 32, 65536, EINVAL), (4, 65568, 32, 65568, EUNSUPPORTED),
    (4, 65536, 32752, 65536, EINVAL), (4, 65536, 32768, 65536, EUNSUPPORTED)])
def test_projection(M, xs, N, K, code):
    assert lib.vitcop_project_mx4(None, xs, A, A, A, N, None, 0, M, N, K, None, 0, None) == code


@pytest.mark.parametrize("M,xs,code", [(1 << 19, 4088, EINVAL), (1 << 19, 4096, EUNSUPPORTED), (1 << 19, WRAPS, EUNSUPPORTED)])
def test_projection_in_bf16(M, xs, code):
    assert lib.vitcop_project(None, xs, A, A, 32, None, 0, M, 32, 64, None, None, 0, None) == code


def test_features_whose_rows_wrap():
    cluster = lambda B, n, rs, bs: lib.vitcop_vic_cluster(A, rs, bs, A, B, n, 64, 8.0, 0.6, 4, A, A, None, None, None, None, None,  # noqa: E731
                                                          0, None)
    merge = lambda B, n, rs, bs: lib.vitcop_collab_prune_merge(A, rs, bs, A, A, A, B, n, 64, 16, A, A, A, None, None, 0, None)      # noqa: E731
    assert cluster(1, 256, (1 << 23) - 8, 0) == EWORKSPACE and cluster(1, 256, 1 << 23, 0) == EUNSUPPORTED
    assert cluster(1, 256, 1 << 56, 0) == EUNSUPPORTED
    for call in (cluster, merge):
        assert call(2, 256, 64, 256 * 64) == EWORKSPACE and call(2, 256, 64, 256 * 64 - 8) == EINVAL
        assert call(2, 256, 1 << 56, 64) == EINVAL


# Four wavefronts to a workgroup of 256 threads: 2^24 workgroups would be 2^32 threads, one more than a launch may have.
@pytest.mark.parametrize("B,Hkv,blocks,code", [(1, 1, (1 << 26) - 4, EINVAL), (1, 1, (1 << 26) - 3, EUNSUPPORTED),
                                               (4, 3, 5592405, EINVAL), (2731, 3, 8191, EUNSUPPORTED), (1, 1, 1 << 26, EUNSUPPORTED)])
def test_rows_of_a_cache(B, Hkv, blocks, code):
    C, T = vc.CacheMx4T(B, 64, Hkv, 128, A, A, A, A), 8 * blocks - 1
    assert T // 8 + 1 == blocks
    assert lib.vitcop_cache_mx4_write(C, None, None, 384, 1024, T, 0, A, None, None) == code
    assert lib.vitcop_cache_mx4_read(C, None, None, T, 0, A, None) == code
