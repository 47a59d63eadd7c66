"""Page operations on the GPU, through the C ABI, against the plain oracle: tables, lengths, counts and every byte of the pages."""
import numpy as np
import pytest
import torch

from oracle.pages_oracle import Pool
from paper_2605_16928_b200 import binding as rb

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Device:
    """The pool of an oracle, on the device: pages filled with random bytes."""

    def __init__(self, pool: Pool, n_kv=2, n_ih=1, kv4=False, ikey8=False, seed=0, kv=True):
        self.pool = pool
        N = len(pool.refs)
        g = torch.Generator(device="cuda").manual_seed(seed)

        def make(*shape, dtype):
            t = torch.randint(0, 256, (N, *shape[:-1], shape[-1] * (2 if dtype == torch.bfloat16 else 1)), dtype=torch.uint8, device="cuda", generator=g)
            return t.view(dtype)

        t = torch.uint8 if kv4 else torch.bfloat16
        self.k, self.v = (make(n_kv, 64, 64 if kv4 else 128, dtype=t) if kv else None for _ in range(2))
        self.s = make(n_kv, 64, 16, dtype=torch.uint8) if kv4 else None
        self.ik = make(n_ih, 64, 16, dtype=torch.uint8 if ikey8 else torch.bfloat16) if n_ih else None
        self.arrays = [x for x in (self.k, self.v, self.s, self.ik) if x is not None]
        self.first = [x.clone() for x in self.arrays]
        self.table, self.lens, self.refs = _i32(pool.table), _i32(pool.lens), _i32(pool.refs)
        self.ctx = rb.Context()
        self.params = rb.Params(n_kv, n_kv, [], [], list(range(min(n_ih, 1))) * n_ih, [])
        self.cache = rb.make_cache(self.k, self.v, self.ik, self.table, self.lens, kv_scales=self.s)
        self.ws = torch.empty(rb.rtp_cache_workspace_bytes(self.cache, pool.table.shape[0]), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.n_used = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.p = (self.ctx, self.params, self.cache)

    def fork(self, src, dst, **kw):
        rb.rtp_cache_fork(*self.p, self.refs, _i32(src), _i32(dst), self.status, **kw)

    def reserve(self, seqs, n, **kw):
        rb.rtp_cache_reserve(*self.p, self.refs, _i32(seqs), _i32(n), self.ws, self.status, **kw)

    def free(self, seqs, **kw):
        rb.rtp_cache_free(*self.p, self.refs, _i32(seqs), self.status, **kw)

    def compact(self, **kw):
        rb.rtp_cache_compact(*self.p, self.refs, self.n_used, self.ws, self.status, **kw)

    def code(self):
        c = rb.rtp_check_status(self.ctx, self.status)
        self.status.zero_()
        return c

    def same(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.table.cpu().numpy(), self.pool.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.pool.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.pool.refs)
        at = torch.from_numpy(self.pool.contents).cuda()
        for x, f in zip(self.arrays, self.first):
            assert torch.equal(x.view(torch.uint8), f[at].view(torch.uint8))


KINDS = [dict(), dict(kv4=True, n_ih=2, ikey8=True, n_kv=3), dict(n_ih=0, n_kv=1), dict(kv=False, n_ih=3)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_random_calls(kind):
    rng = np.random.default_rng(kind)
    pool = Pool(300, 12, 21)
    d = Device(pool, **KINDS[kind])
    for step in range(150):
        seqs = rng.permutation(12)[:rng.integers(1, 7)].tolist()
        what = rng.integers(5)
        pool.invalid = pool.capacity = False
        if what == 0:
            dst = rng.permutation(12)[:len(seqs)].tolist()
            d.fork(seqs, dst), pool.fork(seqs, dst)
        elif what in (1, 2):
            n = rng.integers(0, 400, len(seqs)).tolist()
            d.reserve(seqs, n), pool.reserve(seqs, n)
            if not pool.capacity:
                for s, k in zip(seqs, n):
                    pool.lens[s] += k
                d.lens.copy_(_i32(pool.lens))
        elif what == 3:
            d.free(seqs[:2]), pool.free(seqs[:2])
        else:
            d.compact()
            assert pool.compact() == int(d.n_used)
        assert d.code() == (rb.RTP_ERR_CAPACITY if pool.capacity else rb.RTP_ERR_INVALID if pool.invalid else rb.RTP_OK), step
        d.same()
        pool.check()


@pytest.mark.parametrize("num_pages", [1, 3, 127, 128, 129, 4095, 5000, 32768, 32769, 70001])
def test_pool_sizes(num_pages):
    """The scan over the counts at every kind of pool size, down to a pool of one page, filled to the last page."""
    pool = Pool(num_pages, 3, num_pages + 1)
    d = Device(pool, n_kv=1, n_ih=1, kv=False)
    a = num_pages // 2
    for seqs, n in (([0, 1], [64 * a, 0]), ([1], [64 * (num_pages - a)]), ([2], [1])):
        pool.capacity = False
        d.reserve(seqs, n), pool.reserve(seqs, n)
        assert d.code() == (rb.RTP_ERR_CAPACITY if pool.capacity else rb.RTP_OK)
        if not pool.capacity:
            for s, k in zip(seqs, n):
                pool.lens[s] += k
            d.lens.copy_(_i32(pool.lens))
        d.same()
    assert pool.capacity
    d.free([0]), pool.free([0])
    d.compact()
    assert pool.compact() == int(d.n_used)
    d.same()
    d.compact()                                 # nothing left to move
    pool.compact()
    d.same()
    assert d.code() == rb.RTP_OK


def test_many_sequences_write_one_shared_page():
    """300 samples of one prompt, all listed: all but one of the page's holders get a copy, in the order of the list."""
    n = 300
    pool = Pool(1000, n + 1, 4)
    d = Device(pool, n_kv=1)
    for x in (d, pool):
        x.reserve([0], [100])
    pool.lens[0] = 100
    d.lens.copy_(_i32(pool.lens))
    order = np.random.default_rng(0).permutation(n + 1)
    for x in (d, pool):
        x.fork([0] * n, list(range(1, n + 1)))
        x.reserve(order, [1 + i % 3 * 60 for i in range(n + 1)])
    assert pool.refs[1] == 1 and d.code() == rb.RTP_OK
    d.same()


def test_wrong_requests_are_reported_and_skipped():
    pool = Pool(20, 4, 5)
    d = Device(pool)
    for x in (d, pool):
        x.reserve([0, 9, 1, 0, -1, 2], [70, 1, 64, 5, 5, -3])
    assert pool.invalid and d.code() == rb.RTP_ERR_INVALID
    d.same()
    pool.lens[:2] = 70, 64
    d.lens.copy_(_i32(pool.lens))
    for src, dst in (([0, 0], [2, 2]), ([0, 2], [3, 1]), ([0], [0]), ([2], [2]), ([5, 0], [3, 7])):
        for x in (d, pool):
            x.fork(src, dst)
        assert pool.invalid and d.code() == rb.RTP_ERR_INVALID
        d.same()
        pool.invalid = False
    for x in (d, pool):
        x.free([3, 3, 4, -1, 1])
    assert pool.invalid and d.code() == rb.RTP_ERR_INVALID
    d.same()
    # a row shorter than asked for, for one of two: nothing happens for either
    for x in (d, pool):
        x.reserve([1, 0], [10, 64 * 5])
    assert pool.capacity and d.code() == rb.RTP_ERR_CAPACITY
    d.same()
    # a huge request
    for x in (d, pool):
        x.reserve([1], [2 ** 31 - 1])
    assert d.code() == rb.RTP_ERR_CAPACITY
    d.same()


def test_thousands_of_requests_in_one_call():
    """More requests than the planning block has threads, sharing pages in groups of three."""
    n = 3000
    pool = Pool(9000, n, 3)
    for i in range(0, n, 3):
        pool.table[i:i + 3, 0] = i
        pool.refs[i] = 3
        pool.lens[i:i + 3] = 1 + i % 63
    d = Device(pool, n_kv=1, n_ih=1, kv=False)
    order = np.random.default_rng(0).permutation(n)
    add = np.random.default_rng(1).integers(0, 100, n)
    for x in (d, pool):
        x.reserve(order, add)
    assert d.code() == rb.RTP_OK
    d.same()
    pool.check()


def test_a_shortened_sequence_does_not_write_into_shared_pages():
    """A forked sequence made shorter by its owner: pages behind its end are still the source's, so room in them is refused."""
    pool = Pool(30, 3, 8)
    d = Device(pool)
    for x in (d, pool):
        x.reserve([0], [300])
    pool.lens[0] = 300
    d.lens.copy_(_i32(pool.lens))
    for x in (d, pool):
        x.fork([0], [1])
    for ln, add, ok in ((10, 54, True), (10, 55, False), (64, 1, False), (300, 20, True), (128, 0, True)):
        for x in (d, pool):
            x.free([1])
            x.fork([0], [1])
        pool.lens[1] = ln
        d.lens.copy_(_i32(pool.lens))
        pool.invalid = False
        for x in (d, pool):
            x.reserve([1, 2], [add, 70])
        assert pool.invalid == (not ok) and d.code() == (rb.RTP_OK if ok else rb.RTP_ERR_INVALID)
        d.same()
        pool.check()
        for x in (d, pool):
            x.free([2])


def test_broken_tables_are_reported():
    """Entries that name no page, or a page that nobody holds: reported, and nothing outside the arrays is touched."""
    pool = Pool(40, 3, 4)
    for x in (pool,):
        x.reserve([0, 1], [200, 100])
    d = Device(pool)
    table = d.table.clone()
    d.table[0, 1] = 1 << 20
    d.table[1, 1] = 39                                     # free
    refs = d.refs.clone()
    d.compact()
    assert d.code() == rb.RTP_ERR_INVALID
    assert d.table[0, 1] == 1 << 20 and d.table[1, 1] == 39 and torch.equal(d.refs, refs)
    d.free([0, 1])
    assert d.code() == rb.RTP_ERR_INVALID
    assert (d.table == -1).all() and int(d.refs.sum()) == 2      # the two pages whose entries were overwritten
    d.table.copy_(table)
    d.lens[0] = 130
    d.table[0, 2] = 40                                     # the page that the next token would go to does not exist
    d.reserve([0, 2], [1, 64])
    assert d.code() == rb.RTP_ERR_INVALID and d.table[0, 2] == 40 and d.table[2, 0] >= 0
    d.table[0] = torch.tensor([-1, -1, -1, 3])             # mapped behind an unmapped entry
    d.lens[0] = 0
    d.reserve([0], [256])
    assert d.code() == rb.RTP_ERR_INVALID and d.table[0].tolist() == [-1, -1, -1, 3]
    d.fork([0], [1])                                       # (1 has the pages that were put back above)
    assert d.code() == rb.RTP_ERR_INVALID and torch.equal(d.table[1], table[1])


@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_copy_pages(kind):
    pool = Pool(60, 1, 1)
    d = Device(pool, **KINDS[kind])
    perm = np.random.default_rng(1).permutation(60)
    src, dst = perm[:25], perm[25:50]
    src = np.concatenate([src, src[:5], [7]])                    # a page may be copied to several places, or to itself
    dst = np.concatenate([dst, perm[50:55], [7]])
    if 7 in perm[25:55]:
        src, dst = src[:-1], dst[:-1]
    rb.rtp_cache_copy_pages(*d.p, _i32(src), _i32(dst), d.status)
    pool.contents[dst] = pool.contents[src]
    assert d.code() == rb.RTP_OK
    d.same()
    rb.rtp_cache_copy_pages(*d.p, _i32([60, -1, 3]), _i32([1, 2, 99]), d.status)
    assert d.code() == rb.RTP_ERR_INVALID
    d.same()
    rb.rtp_cache_copy_pages(*d.p, _i32([]), _i32([]), d.status)
    d.same()


def test_captured_step_on_another_stream():
    """A graph that frees, forks and reserves, replayed: each replay starts from the state that the one before left."""
    pool = Pool(64, 5, 6)
    d = Device(pool)
    for x in (d, pool):
        x.reserve([0], [70])
    pool.lens[0] = 70
    d.lens.copy_(_i32(pool.lens))
    src, dst, one = _i32([0, 0, 0]), _i32([1, 2, 3]), _i32([1, 100, 1])

    def step(stream=None):
        rb.rtp_cache_free(*d.p, d.refs, dst, d.status, stream=stream)
        rb.rtp_cache_fork(*d.p, d.refs, src, dst, d.status, stream=stream)
        rb.rtp_cache_reserve(*d.p, d.refs, dst, one, d.ws, d.status, stream=stream)

    def plain():
        pool.free([1, 2, 3])
        pool.fork([0, 0, 0], [1, 2, 3])
        pool.reserve([1, 2, 3], [1, 100, 1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    plain()
    d.same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        plain()
        d.same()
    assert d.code() == rb.RTP_OK


def test_refusals():
    pool = Pool(10, 2, 4)
    d = Device(pool)

    def refused(code, f, *a):
        with pytest.raises(rb.RtpError) as e:
            f(*a)
        assert e.value.code == code
        d.same()

    one = _i32([0])
    refused(rb.RTP_ERR_INVALID, rb.rtp_cache_free, *d.p, None, one, d.status)
    refused(rb.RTP_ERR_INVALID, rb.rtp_cache_free, *d.p, d.refs.data_ptr() + 4, one, d.status)
    refused(rb.RTP_ERR_CAPACITY, rb.rtp_cache_reserve, *d.p, d.refs, one, one, d.ws[:64], d.status)
    refused(rb.RTP_ERR_INVALID, rb.rtp_cache_reserve, *d.p, d.refs, one, one, d.ws[8:], d.status)
    refused(rb.RTP_ERR_CAPACITY, rb.rtp_cache_compact, *d.p, d.refs, d.n_used, d.ws[:64], d.status)
    refused(rb.RTP_ERR_INVALID, rb.rtp_cache_compact, *d.p, d.refs, None, d.ws, d.status)
    many = _i32([0] * 5000)
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_cache_reserve, *d.p, d.refs, many, many, d.ws, d.status)
    params = rb.Params(2, 2, [], [], [0], [1])
    local = rb.make_cache(d.k, d.v, d.ik, d.table, d.lens, d.k, d.v, d.table, 1)
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_cache_free, d.ctx, params, local, d.refs, one, d.status)
    half = rb.make_cache(d.k, None, d.ik, d.table, d.lens)
    refused(rb.RTP_ERR_INVALID, rb.rtp_cache_copy_pages, d.ctx, d.params, half, one, one, d.status)
    assert rb.rtp_cache_workspace_bytes(d.cache, 5000) == 0 and rb.rtp_cache_workspace_bytes(d.cache, -1) == 0


def test_samples_of_a_prompt_decode_like_separate_sequences():
    """The calls as they are used together: room for a prompt, its rows appended to a 4-bit cache, forked, a token of its own
    appended to each sample, attention; then the pool is compacted and attention gives the same bits."""
    from tests import kv4_harness as h
    rng = np.random.default_rng(4)
    n, L = 4, 100
    c = h.Cache4([L + 1] * n, n_kv=2, group=2, ret_kv=(0,), seed=1,
                 k=[rng.standard_normal((L + 1, 2, 128)) for _ in range(n)], v=[rng.standard_normal((L + 1, 2, 128)) for _ in range(n)])
    k, v = rng.standard_normal((2, L + n, 2, 128))
    N, W = 24, 4
    kp, vp = (torch.full((N, 2, 64, 64), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    sp = torch.full((N, 2, 64, 16), 255, dtype=torch.uint8, device="cuda")
    table, lens = torch.full((n + 2, W), -1, dtype=torch.int32, device="cuda"), torch.zeros(n + 2, dtype=torch.int32, device="cuda")
    refs = torch.zeros(N, dtype=torch.int32, device="cuda")
    cache = rb.make_cache(kp, vp, None, table, lens, kv_scales=sp)
    ws = torch.empty(rb.rtp_cache_workspace_bytes(cache, n), dtype=torch.uint8, device="cuda")
    p = (c.ctx, c.params, cache)
    st, n_used = c.status, _i32([0])
    rb.rtp_cache_reserve(*p, refs, _i32([n + 1, n]), _i32([200, L]), ws, st)       # (another sequence in front, freed later)
    rb.rtp_kv_append(*p, h.dev_bf16(k[:L]), h.dev_bf16(v[:L]), _i32([n] * L), _i32(range(L)), st)
    lens[n] = L
    rb.rtp_cache_fork(*p, refs, _i32([n] * n), _i32(range(n)), st)
    rb.rtp_cache_reserve(*p, refs, _i32(range(n)), _i32([1] * n), ws, st)
    rb.rtp_kv_append(*p, h.dev_bf16(k[L:]), h.dev_bf16(v[L:]), _i32(range(n)), _i32([L] * n), st)
    lens[:n] += 1
    for b in range(n):                                                             # what each sample's tokens are
        rows = list(range(L)) + [L + b]
        for name, x in (("k", k), ("v", v)):
            from oracle import kv4_oracle as k4
            from paper_2605_16928_b200 import synth
            getattr(c, name)[b] = k4.decode(*k4.encode(synth.from_bf16(synth.to_bf16(x[rows].astype(np.float32))).astype(np.float64)))
    rb.rtp_dense_attn_decode(*p, *c.args()[3:], None, c.out, c.lse, c.ws, st)
    assert c.code() == rb.RTP_OK
    c.check(range(4), lambda r, hd: range(L + 1))
    first = c.out.clone(), c.lse.clone()
    rb.rtp_cache_free(*p, refs, _i32([n + 1, n]), st)
    rb.rtp_cache_compact(*p, refs, n_used, ws, st)
    assert int(n_used) == 1 + n and not refs[1 + n:].any()                          # one shared page, one of its own each
    rb.rtp_dense_attn_decode(*p, *c.args()[3:], None, c.out, c.lse, c.ws, st)
    assert c.code() == rb.RTP_OK and torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])
