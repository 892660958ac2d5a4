"""CPU test of sizes at the limits that zc.h names for layer norm, embedding and the step for matrices."""
import pytest

import paper_2502_18554_amd as zc

MOST = (1 << 31) - 1


def test_workspaces_at_the_limits():
    for vocab, cols in ((1 << 29, 1), (1, 1), (50000, 1 << 23)):
        for n in (MOST, MOST - 1, 1 << 30):
            assert 8 * n + 4 * vocab <= zc.zc_embedding_workspace_bytes(n, vocab, cols) <= 8 * n + 16 * vocab + (1 << 21) * cols * 4 + (1 << 20)
    assert zc.zc_embedding_workspace_bytes(MOST + 1, 5, 5) == 0
    for cols in (1, 16384, 16385, 1 << 27):
        assert 8 * cols <= zc.zc_layer_norm_workspace_bytes(MOST, cols) <= 8 * 512 * cols + 8 * MOST + 64
    assert zc.zc_layer_norm_workspace_bytes(MOST + 1, 16) == 0


@pytest.mark.parametrize("wide", [False, True])
def test_steps_for_the_largest_sides(wide):
    side, planes = 1 << 20, 2 if wide else 1
    for shape in ((side, 1), (1, side), (side, 1000), (side, side)):
        r, c = min(shape), max(shape)
        along = -(-r // 128) * 128
        least = planes * 2 * (r * c + 2 * c * along + 2 * r * along)
        assert least <= zc.zc_muon_workspace_bytes([shape], wide) <= least + planes * 2 * r * 128 + 8192
        assert zc.zc_muon_state_bytes([shape]) == 4 * -(-r * c // 32) * 32
    assert zc.zc_muon_workspace_bytes([(side + 1, 1)], wide) == 0 and zc.zc_muon_state_bytes([(1, side + 1)]) == 0
