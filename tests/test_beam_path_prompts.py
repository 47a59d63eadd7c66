"""BeamPath.prompts without a device: what it makes of the prompts' lengths, and that it waits for nothing."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild
from paper_2605_16928_b200 import pipeline


@pytest.fixture()
def path(monkeypatch):
    rbuild.build_library()
    monkeypatch.setattr(rb, "Context", lambda: None)
    pool = pipeline.PagePool(rb.Params(4, 2, [], [], [], []), num_pages=10, batch=6, max_pages=4, device="cpu")
    pool.cache_of(*(torch.zeros((10, 2, 64, 128), dtype=torch.bfloat16) for _ in range(2)))
    monkeypatch.setattr(pool, "reserve", lambda seqs, n: None)
    return pipeline.BeamPath([pool], rb.Rope(torch.zeros(64, dtype=torch.float64)), 2, 3, 100, 20)


def test_the_batch_of_the_prompts(path):
    path.prompts([4, 1])
    seq, start, offsets, tok_seq, tok_pos = (x.tolist() for x in path.batch)
    assert (seq, start, offsets, tok_seq, tok_pos) == ([0, 3], [0, 0], [0, 4, 5], [0, 0, 0, 0, 3], [0, 1, 2, 3, 0])
    assert path.pools[0].seq_lens.tolist() == [4, 0, 0, 1, 0, 0]


def test_nothing_is_read_back(path, monkeypatch):
    """A repetition by counts on the device has to be told its length, or it waits to read it."""
    repeat, sizes = torch.repeat_interleave, []

    def told(x, n, **kw):
        sizes.append(kw.get("output_size"))
        return repeat(x, n, **kw)

    monkeypatch.setattr(torch, "repeat_interleave", told)
    for name in ("item", "tolist", "cpu", "numpy", "__bool__", "__int__", "__index__"):
        monkeypatch.setattr(torch.Tensor, name, lambda *a, **kw: pytest.fail("a tensor is read"))
    path.prompts([9, 11])
    assert all(n == 20 for n in sizes)
