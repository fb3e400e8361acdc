"""What the 16-bit layers choose and refuse near the limits of their sizes: decided on the host, so no GPU is needed."""
import os
import re

import pytest

import paper_2410_13229_amd as Q
from paper_2410_13229_amd import build

P = 1 << 20  # a made-up, aligned address: never touched
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


def test_linattn_cuts_a_prompt_into_as_many_segments_as_the_workspace_holds():
    """80 heads of 128 x 64: four prompts of 2048 tokens ask for nothing, one of them for room for its segments."""
    small, large = (Q.quamba_linattn_workspace_bytes(b, 2048, 1, 80, 128, 64) for b in (4, 1))
    assert small == 256 and large > 1 << 20
    assert Q.quamba_debug_linattn_blocks(4, 2048, 80, 128, 64, small) == 32
    assert Q.quamba_debug_linattn_blocks(1, 2048, 80, 128, 64, large) < 32
    last = 0
    for room in (0, 256, large // 3, large // 2, large - 1, large, 1 << 40):
        blocks = Q.quamba_debug_linattn_blocks(1, 2048, 80, 128, 64, room)
        segments = -(-32 // blocks)
        assert segments >= last  # never fewer with more room
        assert segments == 1 or segments * 80 * (128 * 64 * 4 + 8) <= room
        last = segments
    assert Q.quamba_debug_linattn_blocks(1, 2048, 80, 128, 64, 0) == 32


@pytest.mark.parametrize("M, N, K", [(1, 1 << 26, 2048), (2, 1 << 28, 8), (16, 1 << 27, 7), (4, 1 << 26, 2049)])
def test_linear_refuses_more_columns_than_a_launch_takes(M, N, K):
    """A launch counts its threads in 32 bits."""
    with pytest.raises(Q.QuambaError) as e:
        Q.quamba_linear(Q.TYPE_F16, P, K, P, K, None, None, 0, M, N, K, Q.ACT_NONE, Q.TYPE_F16, P, N, None)
    assert e.value.code == -2 and "more than one launch" in str(e.value)


@pytest.mark.parametrize("Bt, Hv, dv", [(65535, 257, 1), (1 << 14, 1 << 9, 129), (1 << 12, 1 << 12, 1)])
def test_linattn_prefill_refuses_more_workgroups_than_a_launch_takes(Bt, Hv, dv):
    with pytest.raises(Q.QuambaError) as e:
        Q.quamba_linattn_prefill(Q.TYPE_F16, P, Hv, P, Hv, P, Hv * dv, None, 0, None, Bt, 1, Hv, Hv, 1, dv, 1.0, P, Hv * dv, None, None)
    assert e.value.code == -2 and "more than one launch" in str(e.value)


def test_the_direct_to_lds_load_declares_the_register_it_writes():
    """m0 is written inside the statement: a compiler that is not told could take an older value of its own for still there."""
    source = open(os.path.join(os.path.dirname(Q.__file__), "csrc", "linattn.hip")).read()
    statements = re.findall(r"asm volatile\(([^;]*?)\);", source, re.S)
    writes = [s for s in statements if "s_mov_b32 m0" in s]
    assert writes and all(s.rstrip().endswith('"m0"') for s in writes)


def _remarks(name, scratch, vgprs, sgprs):
    return "".join("x.hip:1:1: remark: %s [-Rpass-analysis=kernel-resource-usage]\n" % r for r in (
        "Function Name: " + name, "    ScratchSize [bytes/lane]: %d" % scratch, "    SGPRs Spill: %d" % sgprs, "    VGPRs Spill: %d" % vgprs))


@pytest.mark.parametrize("name, scratch, vgprs, sgprs, refused", [
    ("_Z21linattn_blocks_kernelIDF16_E", 52, 16, 90, True), ("_Z21linattn_blocks_kernelIDF16_E", 0, 2, 0, True),
    ("_Z21linattn_blocks_kernelIDF16_E", 0, 0, 90, False), ("_Z17linear_dma_kernelIDF16_E", 0, 0, 1, True),
    ("_Z17linear_dma_kernelIDF16_E", 0, 0, 0, False), ("_Z19linattn_step_kernelIDF16_E", 8, 2, 70, False)])
def test_the_build_refuses_scratch_memory_where_loads_are_counted(name, scratch, vgprs, sgprs, refused):
    if refused:
        with pytest.raises(RuntimeError, match="spills"):
            build._check_spills(_remarks(name, scratch, vgprs, sgprs))
    else:
        build._check_spills(_remarks(name, scratch, vgprs, sgprs))
