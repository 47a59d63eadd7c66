"""rtp_attn_chunks against 64 bits: ragged batches, group sizes, patterns, pools, cuts along the keys, and what it refuses."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Batch:
    """Sequences in a paged cache whose unused places hold NaN, and chunks of their rows."""

    def __init__(self, lens, chunks, n_kv=2, group=2, local=(), ret=(), window=70, n_sink=4, seed=0, ring=None, extra_rows=3, cols=0, scale=1.0):
        """chunks: (sequence, first position, rows)."""
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.lens, self.chunks, self.n_kv, self.G, self.local = list(lens), list(chunks), n_kv, group, list(local)
        self.n_q, self.window, self.n_sink, self.ret = n_kv * group, window, n_sink, list(ret)
        pages = [-(-n // 64) for n in lens]
        W, N = max(max(pages), 1, cols), sum(pages) + 2
        perm = torch.randperm(N, generator=torch.Generator().manual_seed(seed))
        table = torch.full((len(lens), W), -1, dtype=torch.int32)
        at = 0
        self.k, self.v = [], []
        main = [h for h in range(n_kv) if ring is None or h not in self.local]
        kp, vp = (torch.full((N, max(1, len(main)), 64, 128), torch.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        a = {}
        if ring is not None:
            lt = torch.arange(len(lens) * (1 + ring), dtype=torch.int32, device=DEV).reshape(len(lens), 1 + ring)
            lk, lvp = (torch.full((lt.numel(), len(self.local), 64, 128), torch.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            a = dict(k_local_pages=lk, v_local_pages=lvp, local_block_table=lt, sink_pages=1)
        for b, n in enumerate(lens):
            k, v = (scale * torch.randn((n, n_kv, 128), device=DEV, generator=g).bfloat16() if x == 0 else torch.randn((n, n_kv, 128), device=DEV, generator=g).bfloat16()
                    for x in range(2))
            self.k.append(k.float().cpu().numpy())
            self.v.append(v.float().cpu().numpy())
            table[b, :pages[b]] = perm[at:at + pages[b]].int()
            t = torch.arange(n, device=DEV)
            phys = perm[at:at + pages[b]].to(DEV)[t // 64]
            at += pages[b]
            for i, h in enumerate(main):
                kp[phys, i, t % 64], vp[phys, i, t % 64] = k[:, h], v[:, h]
            if ring is not None:
                entry = torch.where(t // 64 < 1, t // 64, 1 + (t // 64 - 1) % ring)
                for i, h in enumerate(self.local):
                    for lo in range(0, n, 64):   # in order: later tokens replace earlier ones
                        s = slice(lo, min(n, lo + 64))
                        lk[lt[b].long()[entry[s]], i, t[s] % 64], lvp[lt[b].long()[entry[s]], i, t[s] % 64] = k[s, h], v[s, h]
        self.table, self.d_lens = table.to(DEV), i32(self.lens)
        self.pages = (kp, vp, a)
        self.ctx = rb.Context()
        self.params = rb.Params(self.n_q, n_kv, self.ret, [0] * len(self.ret), [0] if self.ret else [], self.local, n_sink=n_sink, window=window)
        self.cache = rb.make_cache(kp, vp, None, self.table, self.d_lens, **a)
        off = np.concatenate([[0], np.cumsum([r for _, _, r in self.chunks])])
        self.R = int(off[-1]) + extra_rows
        self.q = torch.randn((self.R, self.n_q, 128), device=DEV, generator=g).bfloat16()
        self.seq, self.start, self.off = i32([c[0] for c in self.chunks]), i32([c[1] for c in self.chunks]), i32(off)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.new_outputs()
        self.ws = torch.empty(rb.rtp_chunk_workspace_bytes(self.params, len(self.chunks), self.R), dtype=torch.uint8, device=DEV)

    def new_outputs(self):
        self.out = torch.full((self.R, self.n_q, 128), 77.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((self.R, self.n_q), 77.0, device=DEV)

    def run(self, pattern=rb.RTP_CHUNK_DENSE, kv_heads=None, stream=None):
        rb.rtp_attn_chunks(self.ctx, self.params, self.cache, self.q, self.seq, self.start, self.off, pattern, kv_heads, self.out, self.lse, self.ws,
                           self.status, stream=stream)

    def code(self):
        c = rb.rtp_check_status(self.ctx, self.status)
        self.status.zero_()
        return c

    def written(self, pattern, kv_heads=None):
        """Query head -> its window (0: everything before the row)."""
        heads = {}
        for h in range(self.n_q):
            kv = h // self.G
            if kv_heads is not None and kv not in kv_heads:
                continue
            loc = kv in self.local
            if pattern == rb.RTP_CHUNK_DENSE or (pattern == rb.RTP_CHUNK_BY_HEAD and (not loc or h in self.ret)):
                heads[h] = 0
            elif loc and pattern != rb.RTP_CHUNK_DENSE and h not in self.ret:
                heads[h] = self.window
        return heads

    def check(self, pattern=rb.RTP_CHUNK_DENSE, kv_heads=None, rows=None, heads=None):
        """rows: at most that many of each chunk (the first and last among them)."""
        out, lse, q = self.out.float().cpu().numpy(), self.lse.cpu().numpy(), self.q.float().cpu().numpy()
        want = self.written(pattern, kv_heads)
        assert all((out[:, h] == 77).all() and (lse[:, h] == 77).all() for h in range(self.n_q) if h not in want)
        at = 0
        for s, p0, r in self.chunks:
            pick = np.arange(r) if rows is None or r <= rows else np.unique(np.linspace(0, r - 1, rows).astype(int))
            for h in want if heads is None else [h for h in heads if h in want]:
                k, v = self.k[s][:, h // self.G], self.v[s][:, h // self.G]
                o, l, mag = og.attend(q[at + pick, h], k, v, p0 + pick, 128 ** -0.5, want[h], self.n_sink)
                got, gl = out[at + pick, h], lse[at + pick, h]
                # P is rounded to bf16 (2^-8 of each probability, so 2^-8 of the mean magnitude), the output once more (2^-8 of it); logits are
                # 32-bit sums of 128 exact products: 130 x 2^-24 of |q| |k| / sqrt(128), and exponents of 2 add 2^-21
                norm = np.linalg.norm(q[at + pick, h], axis=-1) * (np.linalg.norm(k, axis=-1).max() if len(k) else 0) * 128 ** -0.5
                dz = norm * 130 * 2.0 ** -24 + 2.0 ** -20
                tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.2 * dz[:, None]) * mag + 1e-30
                assert (np.abs(got - o) <= tol).all(), (s, p0, r, h, (np.abs(got - o) / tol).max())
                fin = np.isfinite(l)
                assert (gl[~fin] == -np.inf).all() and (np.abs(gl - l)[fin] <= dz[fin] + 2.0 ** -22 * np.abs(l[fin])).all(), (s, p0, r, h)
            at += r
        assert (out[at:] == 77).all() and (lse[at:] == 77).all()   # rows behind the last chunk


@pytest.mark.parametrize("lens,chunks", [
    ([1], [(0, 0, 1)]), ([7], [(0, 0, 7)]), ([200], [(0, 193, 7)]), ([129, 128, 64], [(0, 128, 1), (1, 0, 128), (2, 63, 1)]),
    ([300, 65, 500], [(2, 100, 400), (0, 299, 1), (1, 60, 5)]), ([257], [(0, 0, 257)]), ([640], [(0, 255, 130)]),
])
@pytest.mark.parametrize("n_kv,group", [(2, 1), (1, 4), (3, 3), (2, 8)])
def test_batches(lens, chunks, n_kv, group):
    b = Batch(lens, chunks, n_kv, group, seed=len(lens) + group)
    b.run()
    assert b.code() == rb.RTP_OK
    b.check(rows=40)


@pytest.mark.parametrize("group", [5, 6, 7, 12, 16, 33, 64, 128])
def test_group_sizes(group):
    b = Batch([150, 40], [(0, 100, 50), (1, 38, 2)], 1, group, seed=group)
    b.run()
    assert b.code() == rb.RTP_OK
    b.check(rows=6)


@pytest.mark.parametrize("lens,chunks,n_kv,group", [
    ([20000], [(0, 19999, 1)], 1, 1), ([20000], [(0, 19995, 5)], 2, 4), ([9000, 3, 5000], [(0, 8800, 200), (1, 0, 3), (2, 4999, 1)], 1, 4),
    ([6000], [(0, 5000, 1000)], 1, 2), ([3000] * 5, [(i, 2990 - i, 3) for i in range(5)], 8, 2),
])
def test_sequences_cut_along_their_keys(lens, chunks, n_kv, group):
    b = Batch(lens, chunks, n_kv, group, seed=7)
    b.run()
    assert b.code() == rb.RTP_OK
    b.check(rows=9)
    first = b.out.clone()
    b.new_outputs()
    b.run()
    assert torch.equal(first, b.out)      # the same cut, the same bits


@pytest.mark.parametrize("n", [40, 700])
def test_many_chunks(n):
    """More units than CTAs several times over: whole ones first, then the rest in pieces."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(1, 400, n)]
    chunks = [(int(s), lens[s] - r, r) for s in rng.permutation(n) for r in [int(rng.integers(0, min(lens[s], 70) + 1))]]
    b = Batch(lens, chunks, 8 if n < 100 else 2, 2, seed=n)
    b.run()
    assert b.code() == rb.RTP_OK
    b.check(rows=3, heads=[0, 3, 15])


@pytest.mark.parametrize("window,n_sink", [(1, 0), (70, 4), (128, 0), (129, 200), (64, 128), (5000, 4)])
@pytest.mark.parametrize("pattern", [rb.RTP_CHUNK_LOCAL, rb.RTP_CHUNK_BY_HEAD])
def test_windows(window, n_sink, pattern):
    b = Batch([700, 90, 1000], [(0, 300, 400), (1, 0, 90), (2, 999, 1), (2, 600, 33)], 3, 2, local=[0, 2], window=window, n_sink=n_sink, seed=window)
    b.run(pattern)
    assert b.code() == rb.RTP_OK
    b.check(pattern, rows=25)


def test_mixed_groups_and_chosen_heads():
    b = Batch([500, 300], [(0, 400, 100), (1, 299, 1)], 4, 2, local=[1, 3], ret=[2, 4, 5], window=50, seed=3)
    for pattern, heads in ((rb.RTP_CHUNK_BY_HEAD, None), (rb.RTP_CHUNK_LOCAL, None), (rb.RTP_CHUNK_LOCAL, [3, 0]), (rb.RTP_CHUNK_DENSE, [2]),
                           (rb.RTP_CHUNK_BY_HEAD, [1])):
        b.new_outputs()
        b.run(pattern, heads)
        assert b.code() == rb.RTP_OK
        b.check(pattern, heads, rows=12)


@pytest.mark.parametrize("ring", [5, 9])
def test_truncated_cache(ring):
    b = Batch([1500, 64, 900], [(0, 1440, 60), (1, 0, 64), (2, 899, 1)], 3, 2, local=[1, 2], window=100, ring=ring, seed=ring)
    b.run(rb.RTP_CHUNK_LOCAL)
    assert b.code() == rb.RTP_OK
    b.check(rb.RTP_CHUNK_LOCAL, rows=20)
    b.new_outputs()
    b.run(rb.RTP_CHUNK_BY_HEAD)
    assert b.code() == rb.RTP_OK
    b.check(rb.RTP_CHUNK_BY_HEAD, rows=20)
    b.new_outputs()
    b.run(rb.RTP_CHUNK_DENSE, [0])
    assert b.code() == rb.RTP_OK
    b.check(rb.RTP_CHUNK_DENSE, [0], rows=20)
    with pytest.raises(rb.RtpError) as e:
        b.run(rb.RTP_CHUNK_DENSE)
    assert e.value.code == rb.RTP_ERR_UNSUPPORTED


def test_a_ring_that_is_too_short_is_reported():
    b = Batch([1500, 200], [(0, 1300, 200), (1, 190, 10)], 2, 1, local=[1], window=100, ring=4, seed=1)
    b.run(rb.RTP_CHUNK_LOCAL)
    assert b.code() == rb.RTP_ERR_CAPACITY
    assert (b.out[:200] == 77).all()
    b.chunks = b.chunks[1:]
    out = b.out[200:210, 1].float().cpu().numpy()
    want, _, mag = og.attend(b.q[200:210, 1].float().cpu().numpy(), b.k[1][:, 1], b.v[1][:, 1], range(190, 200), 128 ** -0.5, 100, 4)
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mag).all()


def test_large_logits_and_equal_keys():
    b = Batch([900], [(0, 700, 200)], 1, 2, seed=5, scale=30.0)          # nearly one-hot rows, references that are raised often
    b.run()
    assert b.code() == rb.RTP_OK
    b.check(rows=50)


def test_rows_that_see_nothing_and_positions_that_are_not_there():
    """Lengths of zero, positions beyond the end, sequences out of range; wrong offsets leave rows alone."""
    b = Batch([0, 100, 50], [(0, 0, 3), (1, 90, 20), (2, 45, 5)], 2, 2, seed=9)
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID                                  # (the first two reach beyond their sequences)
    assert (b.out[:3] == 0).all() and torch.isneginf(b.lse[:3]).all()
    b.check()                                                              # (rows beyond the end see all the keys there are)
    b.new_outputs()
    b.seq = i32([0, 7, -1])
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID and (b.out[:28] == 0).all() and (b.out[28:] == 77).all()
    b.new_outputs()
    b.seq, b.start = i32([1, 1, 2]), i32([-5, 0, 45])
    b.off = i32([0, 3, 2, 7])                                              # the second chunk runs backwards
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID and (b.out[:2] == 0).all() and (b.out[7:] == 77).all() and (b.out[2:7] != 77).any()   # (row 2 is named twice)
    b.new_outputs()
    b.off = i32([0, 3, 23, 1000])
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID and (b.out[23:] == 77).all()
    b.new_outputs()
    b.off = i32([0, 28, 0, 28])                                            # more rows in all than the call has
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID
    b.new_outputs()
    b.seq, b.start, b.off = i32([0, 1, 2]), i32([0, 0, 2147483640]), i32([0, 0, 0, 20])
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID
    b.new_outputs()
    b.off = i32([0, 0, 0, 0])
    b.run()
    assert b.code() == rb.RTP_OK and (b.out == 77).all()


def test_queries_that_are_no_numbers_stay_among_themselves():
    b = Batch([300, 9000], [(0, 290, 10), (1, 8998, 2)], 2, 2, seed=2)
    b.run()
    want = b.out.clone()
    b.new_outputs()
    b.q[3, 1, 5] = torch.nan
    b.q[11, 0, :] = torch.nan
    b.run()
    bad = torch.zeros((b.R, b.n_q), dtype=torch.bool, device=DEV)
    bad[3, 1] = bad[11, 0] = True
    assert torch.isnan(b.out[bad]).all() and torch.isnan(b.lse[bad]).all() and torch.equal(b.out[~bad], want[~bad])


def test_a_page_that_is_no_page_is_reported():
    b = Batch([300], [(0, 290, 10)], 1, 1, seed=2)
    b.table[0, 1] = 10 ** 6
    b.run()
    assert b.code() == rb.RTP_ERR_INVALID


def test_the_prefill_call_agrees_on_a_long_chunk():
    b = Batch([5000], [(0, 3000, 2000)], 2, 4, extra_rows=0, seed=11)
    b.run()
    out, lse = torch.zeros_like(b.out), torch.zeros_like(b.lse)
    rb.rtp_dense_attn_prefill(b.ctx, b.params, b.cache, b.q, 0, 3000, 2000, None, out, lse, b.status)
    assert b.code() == rb.RTP_OK
    b.check(rows=30)
    # two results that each are within the bounds of one (P and the output rounded: 2^-8 of magnitudes that are below 1 here)
    assert (b.out.float() - out.float()).abs().max() <= 4 * 2.0 ** -8 and (b.lse - lse).abs().max() <= 2.0 ** -10


def test_captured_replayed_and_on_two_streams():
    a = Batch([3000, 70], [(0, 2990, 10), (1, 69, 1)], 2, 4, seed=1)
    b = Batch([800, 900], [(0, 500, 300), (1, 899, 1)], 2, 4, seed=2)
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = []
    for x, st in zip((a, b), side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            x.run()
        graphs.append(g)
    torch.cuda.synchronize()
    for step in range(3):
        for x, st, g in zip((a, b), side, graphs):
            with torch.cuda.stream(st):
                x.q.mul_(0.5 + step)
                g.replay()
        torch.cuda.synchronize()
    for x in (a, b):
        assert x.code() == rb.RTP_OK
        x.check(rows=10)
    # another batch through the same graph: what a call does is decided on the device
    a.start.copy_(i32([2900, 60]))
    a.chunks = [(0, 2900, 10), (1, 60, 1)]
    graphs[0].replay()
    torch.cuda.synchronize()
    a.check(rows=10)


def test_a_wait_that_runs_out_is_reported():
    b = Batch([500], [(0, 300, 200)], 2, 2, seed=1)
    b.run()
    want = b.out.clone()
    rb.rtp_debug_wait_test(b.ctx, 20_000_000, True)
    b.run()
    assert b.code() == rb.RTP_ERR_TIMEOUT
    rb.rtp_debug_wait_test(b.ctx, 2_000_000_000, False)
    b.new_outputs()
    b.run()
    assert b.code() == rb.RTP_OK and torch.equal(b.out, want)


def test_refusals():
    b = Batch([100], [(0, 90, 10)], 2, 2, local=[1])
    heads = (ctypes.c_int32 * 2)(1, 1)

    def call(**over):
        a = dict(q=b.q.data_ptr(), s=b.seq.data_ptr(), st=b.start.data_ptr(), o=b.off.data_ptr(), n=1, R=b.R, pat=0, kv=None, nh=0, out=b.out.data_ptr(), lse=None,
                 ws=b.ws.data_ptr(), bytes=b.ws.nbytes)
        a.update(over)
        return b.ctx.lib.rtp_attn_chunks(b.ctx.h, b.params.ref(), ctypes.byref(b.cache), *a.values(), b.status.data_ptr(), None)

    assert call() == rb.RTP_OK and call(n=0) == rb.RTP_OK and call(R=0) == rb.RTP_OK
    for over in (dict(q=None), dict(s=None), dict(st=None), dict(o=None), dict(out=None), dict(ws=None), dict(n=-1), dict(R=-1), dict(pat=3), dict(pat=-1),
                 dict(q=b.q.data_ptr() + 8), dict(kv=heads, nh=2), dict(kv=heads, nh=-1), dict(out=b.q.data_ptr())):
        assert call(**over) == rb.RTP_ERR_INVALID, over
    assert call(n=8193) == call(R=1 << 30) == rb.RTP_ERR_UNSUPPORTED
    assert call(bytes=b.ws.nbytes // 2) == rb.RTP_ERR_CAPACITY
    assert rb.rtp_chunk_workspace_bytes(b.params, 0, 5) == rb.rtp_chunk_workspace_bytes(b.params, 5, 0) == rb.rtp_chunk_workspace_bytes(b.params, 8193, 5) == 0
    assert b.code() == rb.RTP_OK
