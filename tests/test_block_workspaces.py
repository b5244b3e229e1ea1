"""Workspaces of the block-scaled FP8 calls: one that is sized for the largest batch serves the
smaller ones, across the sizes where the experts' forms change."""
import pytest

from paper_2602_07265_amd import xshare as X

LAYERS = [(8, 2, 1024, 1408), (1, 1, 2048, 8192), (8, 2, 4096, 14336), (128, 8, 2048, 768),
          (256, 8, 7168, 2048), (1024, 1, 16, 16), (1000, 3, 64, 48), (1, 32, 16, 1024),
          (5, 4, 96, 8208), (90, 2, 16400, 128), (95, 1, 128, 128), (96, 1, 128, 128),
          (3, 3, 16, 12288), (2, 1, 32768, 32768)]


@pytest.mark.parametrize("E,k,d,f", LAYERS)
def test_experts_workspace_never_shrinks(E, k, d, f):
    sizes = [X.block_experts_workspace_bytes(T, k, E, d, f) for T in range(1, 3000)]
    assert sizes[0] > 0
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    # xshare_block_experts' regions: the least that T tokens need
    for T, size in enumerate(sizes, 1):
        assert size >= T * d + T * k * (f + 4 * d + 4)


@pytest.mark.parametrize("n,k", [(100, 272), (4096, 7168)])
def test_linear_workspace_never_shrinks(n, k):
    sizes = [X.block_linear_workspace_bytes(T, n, k) for T in range(1, 3000)]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
