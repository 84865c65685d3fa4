"""Sizes of the workspaces on the host: each has room for its data behind the header and the
completion counters of the calls with many workgroups."""

import pytest

import paper_1802_01561_amd as vt
from paper_1802_01561_amd._lib import CLIP_WORKSPACE_BYTES, lib

HEADER, COUNTERS = 256, 4096


@pytest.mark.parametrize("T,B", [(1, 1), (100, 32), (20, 1000)])
def test_every_kind_leaves_room_for_the_counters(T, B):
    L, A, H, V = lib(), 9, 64, 1000
    front = HEADER + COUNTERS
    assert L.vtrace_workspace_bytes(T, B, A) == front + 24 * B
    assert L.vtrace_head_workspace_bytes(T, B, A, H) >= front + min(B, 512) * (24 + 4 * 16 * (H + 1))
    assert vt.vtrace_vocab_workspace_bytes(T, B, V, H) >= front + 4 * T * B
    assert vt.vtrace_vocab_grad_workspace_bytes(T, B, V, H) >= front + 4 * T * B
    assert vt.vtrace_log_prob_workspace_bytes(T, B) >= front + 24
    assert CLIP_WORKSPACE_BYTES >= front + 8
