"""BeamPath refuses pools that its attention cannot read."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild
from paper_2605_16928_b200 import pipeline


def test_pools_of_four_bits_are_refused(monkeypatch):
    rbuild.build_library()
    monkeypatch.setattr(rb, "Context", lambda: None)
    pools = []
    for fp4 in (False, True):
        pool = pipeline.PagePool(rb.Params(4, 2, [], [], [], []), num_pages=10, batch=6, max_pages=4, device="cpu")
        kv = [torch.zeros((10, 2, 64, 64 if fp4 else 128), dtype=torch.uint8 if fp4 else torch.bfloat16) for _ in range(2)]
        pool.cache_of(*kv, kv_scales=torch.zeros((10, 2, 64, 16), dtype=torch.uint8) if fp4 else None)
        pools.append(pool)
    rope = rb.Rope(torch.zeros(64, dtype=torch.float64))
    pipeline.BeamPath(pools[:1], rope, 2, 3, 100, 20)
    for some in (pools, pools[1:]):
        with pytest.raises(rb.RtpError) as e:
            pipeline.BeamPath(some, rope, 2, 3, 100, 20)
        assert e.value.code == rb.RTP_ERR_UNSUPPORTED
