"""What the 16-bit layers choose and refuse near the limits of their sizes: decided on the host, so no GPU is needed."""
import pytest

import paper_2410_13229_amd as Q

COPY_X, COPY_W = 16, 32
LONG = 1 << 21  # elements of a row from which a tile's rows may not lie within 2^31 bytes


def _room(M, N, K):
    return 2 * (M + N) * (K + 64) + 512


@pytest.mark.parametrize("M, N", [(17, 33), (32, 32), (64, 600), (500, 1100), (2048, 10240), (1 << 14, 1 << 13)])
def test_rows_too_long_for_the_tile_kernels_are_not_copied(M, N):
    """A copy is as long as the row: from 2^21 elements on it would be read with offsets past 31 bits."""
    for K, ld in ((LONG, LONG), (LONG - 63, LONG - 63), (LONG + 8, LONG + 8), (1 << 25, 1 << 25), (35000008, 35000008), (1 << 30, 1 << 30)):
        assert Q.quamba_debug_linear_kind(M, N, K, ld, ld, _room(M, N, K)) in (0, 1)
        assert Q.quamba_linear_workspace_bytes(M, N, K) == 256  # nothing to make room for
    for K, ld in ((LONG - 64, LONG - 63), (LONG - 71, LONG - 71), (1000, LONG), (1000, 1 << 30)):
        kind = Q.quamba_debug_linear_kind(M, N, K, ld, ld, _room(M, N, K))
        assert kind - COPY_X - COPY_W >= 3, kind  # copied, then a tile kernel
        assert Q.quamba_debug_linear_kind(M, N, K, ld, ld, 0) in (0, 1)
    assert Q.quamba_debug_linear_kind(M, N, LONG - 8, LONG - 8, LONG - 8, 0) >= 3  # rows on 16 bytes need no copy


def test_only_what_needs_a_copy_is_copied():
    assert Q.quamba_debug_linear_kind(64, 96, 136, 136, 137, _room(64, 96, 136)) >= COPY_W
    assert COPY_X <= Q.quamba_debug_linear_kind(64, 96, 136, 137, 136, _room(64, 96, 136)) < COPY_W
    assert Q.quamba_debug_linear_kind(64, 96, LONG, 1 << 22, LONG, 1 << 40) == 0  # x and W alike
    assert Q.quamba_debug_linear_kind(16, 96, 135, 135, 135, 1 << 20) == 2  # few rows stream
