"""Workspaces of the gated delta rule on the CPU: what a chunk takes in the calls that need the most for one."""
import pytest

from test_abi import _lib

KB = 1024


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_largest_workspace_of_a_chunk(dtype):
    """128 x 128, tokens that fill their chunks: products and weights 22 KB, the states and gradients 128, errors 32 (bf16: dv's rest 16,
    and with 32-bit outs dv 16), two gradients of a group's heads in pieces 64 each for two heads in one group, two segment states of
    64 KB a chunk where segments are of two; fp32: a boundary of 64 where each chunk has one; bf16: a last state a row."""
    bwd = _lib().packmamba_delta_rule_bwd_workspace_size
    largest = {0: 382, 1: 342, 2: 358}[dtype]
    for B, H, G in ((1, 1, 1), (1, 2, 1), (1, 2, 2), (1, 8, 1), (1, 32, 1), (4, 4, 1), (8, 16, 1), (2, 64, 4)):
        for chunks in (*range(2, 40), 64, 100, 128, 256, 300):
            assert 0 < bwd(B, H, G, 128, 128, 64 * chunks, dtype) <= B * H * chunks * largest * KB, (B, H, G, chunks)
    assert bwd(1, 2, 1, 128, 128, 576, dtype) > 18 * (largest - 4) * KB
    for shape in ((1, 16, 16, 128, 128, 1 << 22), (16, 16, 1, 128, 128, 1 << 18)):      # the most chunks that a call may have
        assert 0 < bwd(*shape, dtype) <= (1 << 20) * 215 * KB, shape
