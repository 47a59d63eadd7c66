"""rtp_attn_chunks on a truncated cache, for chunks that are not their sequence's end: what has been appended behind a chunk has taken
the places of its window's oldest keys in the ring."""
import numpy as np
import pytest

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_chunks import Batch

pytestmark = pytest.mark.gpu
WINDOW, SINKS = 100, 4


def compare(b, pattern, done):
    """The chunks of `done` (a truth value each) against 64 bits; the others' rows as they were."""
    out, q, at = b.out.float().cpu().numpy(), b.q.float().cpu().numpy(), 0
    for (s, p0, r), is_done in zip(b.chunks, done):
        if not is_done:
            assert (out[at:at + r] == 77).all(), (s, p0, r)
        pick = np.unique(np.linspace(0, r - 1, min(r, 24)).astype(int))
        for h, window in b.written(pattern).items() if is_done else ():
            k, v = b.k[s][:, h // b.G], b.v[s][:, h // b.G]
            o, _, mag = og.attend(q[at + pick, h], k, v, p0 + pick, 128 ** -0.5, window, SINKS)
            # P and the output are rounded to bf16 (2^-8 each), logits are 32-bit sums of 128 products (130 x 2^-24 of |q| |k| / sqrt(128))
            dz = np.linalg.norm(q[at + pick, h], axis=-1) * np.linalg.norm(k, axis=-1).max() * 128 ** -0.5 * 130 * 2.0 ** -24 + 2.0 ** -20
            assert (np.abs(out[at + pick, h] - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.2 * dz[:, None]) * mag + 1e-30).all(), (s, p0, r, h)
        at += r
    assert (out[at:] == 77).all()


# one sink page; a chunk needs the ring to hold its window, everything behind its first row, and a page: 100 + (length - start) + 64
@pytest.mark.parametrize("pattern", [rb.RTP_CHUNK_LOCAL, rb.RTP_CHUNK_BY_HEAD])
@pytest.mark.parametrize("lens,chunks,ring,done", [
    ([1500], [(0, 1300, 60)], 6, [True]), ([1500], [(0, 1300, 60)], 5, [False]), ([1500], [(0, 600, 60)], 5, [False]),
    ([1500], [(0, 1300, 60), (0, 1490, 10)], 6, [True, True]), ([1500], [(0, 1300, 60), (0, 1490, 10)], 5, [False, True]),
    ([1500, 300], [(0, 1499, 1), (0, 1450, 50), (0, 1449, 1), (1, 0, 300)], 4, [True, True, True, True]),
    ([1500], [(0, 100, 200)], 4, [False]),                       # the chunk's end lies within the pool, its sequence's does not
    ([320, 321], [(0, 100, 20), (1, 100, 20)], 4, [True, False]),   # as long as the pool, and one more
    ([1500, 50], [(0, 0, 1), (0, 1, 1), (1, 0, 50)], 4, [False, False, True]),
    ([700], [(0, 512, 188)], 6, [True]), ([700], [(0, 480, 220)], 6, [True]), ([700], [(0, 479, 221)], 6, [False]),
])
def test_chunks_in_the_middle_of_a_sequence(lens, chunks, ring, done, pattern):
    b = Batch(lens, chunks, 3, 2, local=[1, 2], window=WINDOW, n_sink=SINKS, ring=ring, seed=ring + len(chunks))
    b.run(pattern)
    assert b.code() == (rb.RTP_OK if all(done) else rb.RTP_ERR_CAPACITY)
    compare(b, pattern, done)


def test_rows_beyond_the_end_need_no_more_of_a_ring():
    """Positions beyond the sequence are reported as such; its rows see the keys that there are."""
    b = Batch([1500], [(0, 1490, 300)], 3, 2, local=[1, 2], window=WINDOW, n_sink=SINKS, ring=3, seed=1)
    b.run(rb.RTP_CHUNK_LOCAL)
    assert b.code() == rb.RTP_ERR_INVALID
    compare(b, rb.RTP_CHUNK_LOCAL, [True])
