"""The gated RMSNorm's largest number of features, on the CPU: features are counted in 32 bits in the kernels, and the
sum for dweight has 32 threads a feature in a grid of fewer than 2^32; more is refused before anything is enqueued."""
import pytest

from test_abi import _gpu_visible, _lib

LARGEST = (1 << 27) - 32


@pytest.mark.skipif(_gpu_visible(), reason="fake pointers are only passed where no GPU exists")
@pytest.mark.parametrize("dim,groups", [(LARGEST + 1, 1), (1 << 27, 1), (1 << 27, 8), ((1 << 31) - 1, 1), ((1 << 31) - 4096, 2), (1 << 31, 1)])
def test_too_many_features(dim, groups):
    lib, P = _lib(), 0x10000
    for dtype in (0, 1, 2):
        for seqlen in (1, 3):
            assert lib.packmamba_gated_rmsnorm_fwd(P, P, P, 1e-5, P, P, 1, dim, seqlen, groups, 1, dtype, None) == 2
            assert lib.packmamba_gated_rmsnorm_bwd(P, P, P, P, P, P, P, P, P, 1 << 62, 1, dim, seqlen, groups, 1, dtype, None) == 2
            assert lib.packmamba_gated_rmsnorm_bwd_workspace_size(1, dim, seqlen, groups) == 0


def test_largest_number_of_features():
    assert _lib().packmamba_gated_rmsnorm_bwd_workspace_size(1, LARGEST, 1, 1) == (4 * LARGEST + 255) // 256 * 256
