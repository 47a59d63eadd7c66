"""rtp_attn_chunks with thousands of chunks: plans whose lists do not lie in shared memory."""
import numpy as np
import pytest

from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_chunks import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,n_kv,group", [(4096, 1, 2), (4097, 2, 1), (8192, 1, 3)])
def test_thousands_of_single_rows(n, n_kv, group):
    """Rows, some chunks without any, of a few hundred sequences; descriptions are made anew for each use."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(1, 300, 300)]
    chunks = [(s, int(rng.integers(0, lens[s])), int(rng.random() < 0.9)) for s in rng.integers(0, 300, n).tolist()]
    b = Batch(lens, chunks, n_kv, group, seed=n)
    b.run()
    assert b.code() == rb.RTP_OK
    b.check()


@pytest.mark.parametrize("pattern", [rb.RTP_CHUNK_DENSE, rb.RTP_CHUNK_BY_HEAD])
@pytest.mark.parametrize("long", [[(0, 19999, 1)], [(0, 19999, 1), (1, 15000, 300), (0, 10000, 2)]])
def test_more_cut_units_than_shared_memory_holds(long, pattern):
    """A few long chunks that no CTA should have alone, among more than a thousand short ones: all of them are laid end to end and cut."""
    rng = np.random.default_rng(len(long))
    lens = [20000, 16000] + [int(x) for x in rng.integers(1, 60, 100)]
    short = [(int(s), int(rng.integers(0, lens[s])), 1) for s in rng.integers(2, 102, 1400)]
    chunks = short[:700] + long + short[700:]
    b = Batch(lens, chunks, 2, 2, local=[1], window=70, seed=7)
    b.run(pattern)
    assert b.code() == rb.RTP_OK
    b.check(pattern, rows=7)
    first = b.out.clone()
    b.new_outputs()
    b.run(pattern)
    assert (first == b.out).all()
