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
