"""GPU parity: projections by a matrix in 4 bits on the largest tiles, in one slice of k."""
import pytest

from test_gpu_mx4 import project_check, vc          # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# tiles of 160 rows of x by 256 of the matrix, several rounds of them, K a whole number of steps of 128 and not
@pytest.mark.parametrize("M,N,K", [(1026, 7184, 544), (3644, 2064, 512)])
def test_projection_on_the_largest_tiles(vc, M, N, K):          # noqa: F811
    project_check(vc, M, N, K, residual=M % 4 == 0, seed=11, one_slice=True)
