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


def _page_pool(num_pages, batch, max_pages, kv4, n_ih=1):
    """A PagePool over one KV head with index keys, and what appends a row of ones to a list of sequences."""
    from paper_2605_16928_b200 import pipeline
    params = rb.Params(2, 1, [0] * n_ih, [0] * n_ih, [0] * n_ih, [])
    pool = pipeline.PagePool(params, num_pages=num_pages, batch=batch, max_pages=max_pages)
    w = 64 if kv4 else 128
    t = torch.uint8 if kv4 else torch.bfloat16
    k, v = (torch.zeros((num_pages, 1, 64, w), dtype=t, device="cuda") for _ in range(2))
    scales = torch.zeros((num_pages, 1, 64, 16), dtype=torch.uint8, device="cuda") if kv4 else None
    ik = torch.zeros((num_pages, 1, 64, 16), dtype=torch.bfloat16, device="cuda")
    cache = pool.cache_of(k, v, ik, kv_scales=scales)
    w_k = torch.ones((1, 128, 16), dtype=torch.bfloat16, device="cuda")

    def append(seqs, pos):
        rows = torch.ones((len(seqs), 1, 128), dtype=torch.bfloat16, device="cuda") * (1 + torch.arange(len(seqs), device="cuda"))[:, None, None]
        rb.rtp_kv_append(pool.ctx, params, cache, rows, -rows, _i32(seqs), _i32(pos), pool.status)
        rb.rtp_index_keys(pool.ctx, params, cache, rows, w_k, _i32(seqs), _i32(pos))

    return pool, append, [x for x in (k, v, scales, ik) if x is not None]


@pytest.mark.parametrize("kv4", [False, True])
def test_a_full_pool_keeps_shared_pages_as_they_are(kv4):
    """Samples of a prompt whose reserve finds the pool full: the appends behind it leave the page that they share alone."""
    pool, append, arrays = _page_pool(3, 4, 4, kv4)
    pool.reserve(_i32([0]), _i32([100]))
    append([0] * 100, list(range(100)))
    pool.seq_lens[0] = 100
    pool.fork(_i32([0, 0]), _i32([1, 2]))
    assert rb.rtp_check_status(pool.ctx, pool.status) == rb.RTP_OK
    before = [x.clone() for x in arrays]
    graph = torch.cuda.CUDAGraph()                     # the step of a server: room, then the rows
    seqs, one = _i32([0, 1, 2]), _i32([1, 1, 1])
    rows = torch.ones((3, 1, 128), dtype=torch.bfloat16, device="cuda") * 3
    w_k, pos = torch.ones((1, 128, 16), dtype=torch.bfloat16, device="cuda"), _i32([100, 100, 100])
    with torch.cuda.graph(graph):
        pool.reserve(seqs, one)
        rb.rtp_kv_append(pool.ctx, pool.params, pool.cache, rows, -rows, seqs, pos, pool.status)
        rb.rtp_index_keys(pool.ctx, pool.params, pool.cache, rows, w_k, seqs, pos)
    graph.replay()
    assert rb.rtp_check_status(pool.ctx, pool.status) == rb.RTP_ERR_CAPACITY
    for x, b in zip(arrays, before):
        assert torch.equal(x, b)
    pool.status.zero_()
    pool.free(_i32([2]))                               # one sample leaves: there is room for the others
    rb.rtp_cache_reserve(pool.ctx, pool.params, pool.cache, pool.page_refs, _i32([0, 1]), _i32([1, 1]), pool.workspace, pool.status)
    append([0, 1], [100, 100])
    assert rb.rtp_check_status(pool.ctx, pool.status) == rb.RTP_OK
    table = pool.block_table.tolist()
    assert table[0][0] == table[1][0] and table[0][1] != table[1][1]
    for x, b in zip(arrays, before):
        assert torch.equal(x[table[0][0]], b[table[0][0]])
        own = [x[table[s][1], :, 36] for s in (0, 1)]
        assert own[0].any() and own[1].any()
        assert x.shape[-1] == 64 or not torch.equal(own[0], own[1])      # (rows of ones and twos have the same 4-bit codes)
        for s in (0, 1):
            assert torch.equal(x[table[s][1], :, :36], b[1, :, :36])


def test_appends_only_go_to_pages_that_one_sequence_holds():
    """Counts of zero (not mapped by a reserve), one and two; a cache that does not name its counts is written as before."""
    for kv4 in (False, True):
        pool, append, arrays = _page_pool(4, 3, 2, kv4)
        pool.block_table[:, 0] = _i32([0, 1, 2])
        pool.page_refs.copy_(_i32([0, 1, 2, 0]))
        before = [x.clone() for x in arrays]
        append([0, 1, 2], [5, 5, 5])
        assert rb.rtp_check_status(pool.ctx, pool.status) == rb.RTP_ERR_INVALID
        for x, b in zip(arrays, before):
            assert torch.equal(x[[0, 2, 3]], b[[0, 2, 3]]) and x[1, :, 5].any()
        plain = rb.make_cache(arrays[0], arrays[1], None, pool.block_table, pool.seq_lens, kv_scales=arrays[2] if kv4 else None)
        rows = torch.ones((3, 1, 128), dtype=torch.bfloat16, device="cuda")
        pool.status.zero_()
        rb.rtp_kv_append(pool.ctx, pool.params, plain, rows, rows, _i32([0, 1, 2]), _i32([6, 6, 6]), pool.status)
        assert rb.rtp_check_status(pool.ctx, pool.status) == rb.RTP_OK
        assert all(arrays[0][p, :, 6].any() for p in range(3))
        other = torch.zeros_like(pool.page_refs)
        with pytest.raises(rb.RtpError) as e:
            rb.rtp_cache_free(pool.ctx, pool.params, pool.cache, other, _i32([0]), pool.status)
        assert e.value.code == rb.RTP_ERR_INVALID and pool.block_table[0, 0] == 0


def test_index_keys_are_not_left_behind():
    """A parameter block without index heads does not say how large the index keys of a page are: refused by every page call."""
    pool = Pool(10, 2, 4)
    d = Device(pool, n_kv=2, n_ih=1)
    none = rb.Params(2, 2, [], [], [], [])
    one = _i32([0])
    p = (d.ctx, none, d.cache)
    for f, a in ((rb.rtp_cache_copy_pages, (one, _i32([1]), d.status)), (rb.rtp_cache_fork, (d.refs, one, _i32([1]), d.status)),
                 (rb.rtp_cache_reserve, (d.refs, one, one, d.ws, d.status)), (rb.rtp_cache_free, (d.refs, one, d.status)),
                 (rb.rtp_cache_compact, (d.refs, d.n_used, d.ws, d.status))):
        with pytest.raises(rb.RtpError) as e:
            f(*p, *a)
        assert e.value.code == rb.RTP_ERR_INVALID
        d.same()
    d.cache = rb.make_cache(d.k, d.v, None, d.table, d.lens)
    rb.rtp_cache_copy_pages(d.ctx, none, d.cache, one, _i32([1]), d.status)
    assert d.code() == rb.RTP_OK and torch.equal(d.k[0].view(torch.uint8), d.k[1].view(torch.uint8))


def test_a_full_pool_is_reported_once():
    """Evicting and trying again: the status of the calls since the last look, not of all calls ever."""
    pool, append, _ = _page_pool(3, 3, 4, True)
    pool.reserve(_i32([0]), _i32([128]))
    assert pool.status_code() == rb.RTP_OK
    pool.reserve(_i32([1]), _i32([128]))
    assert pool.status_code() == rb.RTP_ERR_CAPACITY
    assert pool.status_code() == rb.RTP_OK
    pool.free(_i32([0]))
    pool.reserve(_i32([1]), _i32([128]))
    assert pool.status_code() == rb.RTP_OK and (pool.block_table[1, :2] >= 0).all()
    pool.free(_i32([7]))
    pool.reserve(_i32([2]), _i32([1]))
    assert pool.status_code() == rb.RTP_ERR_INVALID
    pool.reserve(_i32([0]), _i32([300]))
    assert pool.status_code() == rb.RTP_ERR_CAPACITY
