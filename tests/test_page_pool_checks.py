"""What PagePool refuses before anything runs on a device (arrays on the CPU, a context that makes no call)."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild
from paper_2605_16928_b200 import pipeline


@pytest.fixture()
def pool(monkeypatch):
    rbuild.build_library()
    monkeypatch.setattr(rb, "Context", lambda: None)
    return pipeline.PagePool(rb.Params(4, 2, [0], [0], [0], [1]), num_pages=10, batch=2, max_pages=4, device="cpu")


def _arrays(n=10, heads=2, ik_heads=1):
    k, v = (torch.zeros((n, heads, 64, 64), dtype=torch.uint8) for _ in range(2))
    return dict(k_pages=k, v_pages=v, ikey_pages=torch.zeros((n, ik_heads, 64, 16), dtype=torch.bfloat16),
                kv_scales=torch.zeros((n, heads, 64, 16), dtype=torch.uint8))


def test_arrays_of_the_pools_size_are_taken(pool):
    cache = pool.cache_of(**_arrays())
    assert cache.num_pages == 10 and cache.batch == 2 and cache.max_pages == 4
    assert pool.cache_of(**{**_arrays(), "ikey_pages": None}).num_pages == 10
    assert pool.cache_of(None, None, torch.zeros((10, 1, 64, 16), dtype=torch.bfloat16)).num_pages == 10


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "ikey_pages", "kv_scales"])
@pytest.mark.parametrize("wrong", [dict(n=11), dict(n=9), dict(heads=3, ik_heads=2), "strided"])
def test_arrays_of_another_size_are_refused(pool, name, wrong):
    """Counts exist for the pool's pages only: a longer array would have pages handed out behind their end."""
    bad = _arrays()[name].transpose(2, 3) if wrong == "strided" else _arrays(**wrong)[name]
    with pytest.raises(rb.RtpError) as e:
        pool.cache_of(**{**_arrays(), name: bad})
    assert e.value.code == rb.RTP_ERR_INVALID and name in str(e.value) and pool.cache is None


def test_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(rb, "Context", lambda: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(rb.RtpError) as e:
        pipeline.PagePool(rb.Params(4, 2, [], [], [], []), num_pages=10, batch=2, max_pages=4, device="cuda:1")
    assert e.value.code == rb.RTP_ERR_INVALID
