"""Tables, counts and requests that are wrong, or a pool that is full: what the page operations then leave as it was."""
import numpy as np
import pytest
import torch

from oracle.pages_oracle import Pool
from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_pages import Device, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,max_pages", [(3, 4), (40, 700), (300, 2000)])
@pytest.mark.parametrize("page", ["gap", "behind", "last", "none", "far"])
def test_compaction_of_a_wrong_table_moves_nothing(batch, max_pages, page):
    """A table entry that names a free page (a gap that a page in use would be moved into, the first page behind those in use,
    the last of the pool) or no page at all, in the last row of the table."""
    N = 40
    pool = Pool(N, batch, max_pages)
    for seqs, n in (([0, 1], [200, 100]),):
        pool.reserve(seqs, n)
    d = Device(pool, n_kv=1, n_ih=1, kv=False)
    for x in (d, pool):
        x.free([0])
    entry = {"gap": 1, "behind": 2, "last": N - 1, "none": N, "far": 2 ** 31 - 1}[page]
    pool.table[batch - 1, max_pages - 1] = entry
    d.table[batch - 1, max_pages - 1] = entry
    d.compact()
    assert pool.compact() == N and pool.invalid
    assert d.code() == rb.RTP_ERR_INVALID and int(d.n_used) == N
    d.same()
    pool.table[batch - 1, max_pages - 1] = -1
    d.table[batch - 1, max_pages - 1] = -1
    d.compact()
    assert pool.compact() == 2 == int(d.n_used) and d.code() == rb.RTP_OK
    d.same()
    pool.check()


def test_room_in_a_page_that_nobody_holds_is_refused():
    """A mapped page whose count is zero, as the partly filled last page of a sequence or as a page reserved behind it: the
    request is skipped, and the page may go to somebody else."""
    for table, refs, ln, add in (([[3, -1]], [], 10, 5), ([[0, 1]], [0], 64, 10), ([[0, 1]], [0], 20, 100), ([[2, -1]], [], 63, 1)):
        pool = Pool(6, 2, 2)
        pool.table[0] = table[0]
        pool.refs[refs] = 1
        pool.lens[0] = ln
        d = Device(pool, n_kv=1, n_ih=1, kv=False)
        for x in (d, pool):
            x.reserve([0, 1], [add, 128])
        assert pool.invalid and d.code() == rb.RTP_ERR_INVALID
        d.same()
        assert pool.table[0].tolist() == table[0] and (pool.table[1] >= 0).all()
