"""Workspace sizes of parameter blocks without retrieval heads: a cache whose heads are all local or all dense."""
from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild


def test_sizes_without_index_heads():
    rbuild.build_library()
    p = rb.Params(8, 2, [], [], [], [0, 1])
    for rows, n in ((1, 1), (3, 1000), (8192, 131072)):
        assert rb.rtp_workspace_bytes(p, rows, n) >= 0
        assert rb.rtp_block_workspace_bytes(p, rows, n) >= 0
    assert rb.rtp_workspace_bytes(p, 8, 32768) > 0


def test_short_contexts_have_room_for_the_splits_of_a_4bit_call():
    """One sequence of 4096 tokens, 8 KV heads in groups of 4: 16 splits of 32 heads, 130 floats each."""
    rbuild.build_library()
    p = rb.Params(32, 8, [], [], [], [])
    assert rb.rtp_workspace_bytes(p, 1, 4096) >= 16 * 32 * 130 * 4
