"""rtp_attn_chunks where a chunk's positions run to the end of 32 bits."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_chunks import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("start", [2147483647, 2147483640, 2147483500, 2147480000, 100000])
@pytest.mark.parametrize("rows", [1, 20, 400])
def test_rows_far_behind_the_end_see_all_the_keys(start, rows):
    b = Batch([50, 900], [(0, start, rows), (1, 890, 10)], 2, 2, local=[1], window=70, n_sink=4, seed=rows)
    for pattern in (rb.RTP_CHUNK_DENSE, rb.RTP_CHUNK_BY_HEAD):
        b.new_outputs()
        b.run(pattern)
        assert b.code() == rb.RTP_ERR_INVALID
        b.check(pattern, rows=30)          # (with sinks and a window: the sinks)
    assert not (b.out[:rows] == 0).all(-1).any()
    assert torch.isfinite(b.lse[:rows]).all() and np.isfinite(og.attend(np.zeros((1, 128)), b.k[0][:, 0], b.v[0][:, 0], [start], 1.0)[1]).all()
