"""rtp_rope_append: rotated queries and keys against 64 bits, everything else bit for bit against the calls it stands for."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Case:
    def __init__(self, lens, n_kv=2, group=2, n_ih=1, fp4=False, e4m3=False, local=(), seed=0, refs=False):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.n_kv, self.n_q, self.n_ih = n_kv, n_kv * group, n_ih
        B, W = len(lens), max(-(-n // 64) for n in lens)
        N = B * W + 2
        perm = torch.randperm(N, device=DEV, generator=g).int()
        self.table, self.lens = perm[:B * W].reshape(B, W).contiguous(), i32(lens)
        n_main = n_kv - len(local)
        self.ctx = rb.Context()
        self.params = rb.Params(self.n_q, n_kv, [], [], [(n_kv - 1 - j) % n_kv for j in range(n_ih)], list(local), n_sink=4, window=70)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        # (the local pool: one sink page and a ring of three)
        self.ltable = torch.arange(B * 4, dtype=torch.int32, device=DEV).reshape(B, 4).flip(0).contiguous() if local else None
        self.fp4, self.e4m3, self.N, self.n_main, self.n_local, self.local_pages = fp4, e4m3, N, n_main, len(local), B * 4
        self.refs = torch.ones(N, dtype=torch.int32, device=DEV) if refs else None

    def cache(self):
        """Empty arrays and their description.  (A pool that no head lives in is described by some address too.)"""
        n_main = max(1, self.n_main)
        last, dt = (64, torch.uint8) if self.fp4 else (128, torch.bfloat16)
        a = dict(k=torch.zeros((self.N, n_main, 64, last), dtype=dt, device=DEV), v=torch.zeros((self.N, n_main, 64, last), dtype=dt, device=DEV))
        a["ik"] = torch.zeros((self.N, max(1, self.n_ih), 64, 16), dtype=torch.uint8 if self.e4m3 else torch.bfloat16, device=DEV)
        if self.fp4:
            a["sc"] = torch.zeros((self.N, n_main, 64, 16), dtype=torch.uint8, device=DEV)
        if self.n_local:
            a["lk"], a["lv"] = (torch.zeros((self.local_pages, self.n_local, 64, last), dtype=dt, device=DEV) for _ in range(2))
            if self.fp4:
                a["lsc"] = torch.zeros((self.local_pages, self.n_local, 64, 16), dtype=torch.uint8, device=DEV)
        c = rb.make_cache(a["k"], a["v"], a["ik"], self.table, self.lens, a.get("lk"), a.get("lv"), self.ltable, 1 if self.n_local else 0,
                          kv_scales=a.get("sc"), kv_local_scales=a.get("lsc"), page_refs=self.refs)
        return a, c

    def code(self):
        c = rb.rtp_check_status(self.ctx, self.status)
        self.status.zero_()
        return c


def rows(T, c, seed, fused=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((T, c.n_q + 2 * c.n_kv, 128), device=DEV, generator=g).bfloat16()
    q, k, v = x[:, :c.n_q], x[:, c.n_q:c.n_q + c.n_kv], x[:, c.n_q + c.n_kv:]
    return (q, k, v) if fused else tuple(t.contiguous() for t in (q, k, v))


def freqs(rd, base=10000.0):
    return base ** (-torch.arange(rd // 2, device=DEV, dtype=torch.float64) * 2 / rd)


def tokens(lens, new):
    return i32(np.repeat(np.arange(len(lens)), new)), i32(np.concatenate([np.arange(n - t, n) for n, t in zip(lens, new)]))


def check_rotated(got, x, pos, rope):
    exact, mag = og.rotate(x.float().cpu().numpy(), pos.cpu().numpy(), rope.freqs.cpu().numpy(), rope.rotary_dim, rope.interleaved, rope.scale)
    # one rounding to bf16 (half a step: 2^-8 of the value), on top of 32-bit arithmetic: the angle's rounding to 32 bits (half turns up to 1:
    # pi 2^-25), two ulp of sine or cosine (2^-23), the scale's product, two products and a sum (2^-24 each) of |a| + |b|: below 2^-21
    tol = 2.0 ** -8 * np.abs(exact) + abs(rope.scale) * mag * 2.0 ** -21 + 1e-38
    err = np.abs(got.float().cpu().numpy() - exact)
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("rd,interleaved,scale", [(128, False, 1.0), (128, True, 1.0), (64, False, 0.5), (96, True, 1.25), (16, False, 1.0), (48, False, -1.0)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([65, 64, 3], [3, 64, 1]), ([700], [500])])
def test_rows_and_pages(lens, new, rd, interleaved, scale):
    c = Case(lens, n_kv=3, group=2, n_ih=2, seed=rd)
    a, cache = c.cache()
    tok_seq, tok_pos = tokens(lens, new)
    T = len(tok_seq)
    q, k, v = rows(T, c, rd + T)
    rope = rb.Rope(freqs(rd), rd, interleaved, scale)
    w_k = torch.randn((2, 128, 16), device=DEV).bfloat16()
    q_out = torch.full((T, c.n_q, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, q_out, w_k, tok_seq, tok_pos, c.status)
    assert c.code() == rb.RTP_OK
    check_rotated(q_out, q, tok_pos, rope)
    at = (c.table[tok_seq.long(), tok_pos.long() // 64].long(), slice(None), tok_pos.long() % 64)
    check_rotated(a["k"][at], k, tok_pos, rope)
    assert torch.equal(a["v"][at], v)
    # index keys are those of the unrotated rows; nothing else is written
    b, plain = c.cache()
    rb.rtp_index_keys(c.ctx, c.params, plain, k[:, [2, 1]].contiguous(), w_k, tok_seq, tok_pos)
    rb.rtp_kv_append(c.ctx, c.params, plain, a["k"][at].contiguous(), v.contiguous(), tok_seq, tok_pos, c.status)
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("pos", [131071, 1048575, 16777217, 2147483583])
def test_far_positions_keep_their_angles(pos):
    """The append is refused there (the table is short), the queries are rotated all the same."""
    c = Case([64])
    _, cache = c.cache()
    q, k, v = rows(1, c, 5)
    rope = rb.Rope(freqs(128, 500000.0))
    q_out = torch.zeros((1, c.n_q, 128), dtype=torch.bfloat16, device=DEV)
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, q_out, None, i32([0]), i32([pos]), c.status)
    assert c.code() == rb.RTP_ERR_INVALID
    check_rotated(q_out, q, i32([pos]), rope)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("local", [(), (0, 2), (0, 1, 2)])
@pytest.mark.parametrize("T", [5, 190])
def test_every_pool_and_format_is_the_separate_calls(fp4, e4m3, local, T):
    lens = [T + 3, 7]
    new = [T - 2, 2]
    c = Case(lens, n_kv=3, group=1, n_ih=2, fp4=fp4, e4m3=e4m3, local=local, seed=T)
    a, cache = c.cache()
    tok_seq, tok_pos = tokens(lens, new)
    q, k, v = rows(T, c, T)
    rope = rb.Rope(freqs(96), 96)
    w_k = torch.randn((2, 128, 16), device=DEV).bfloat16()
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, None, k, v, None, w_k, tok_seq, tok_pos, c.status)
    assert c.code() == rb.RTP_OK
    # the rotated keys on their own: the call's queries, taken from the keys
    d = Case(lens, n_kv=3, group=1, n_ih=0, seed=T)
    k_rot = torch.zeros((T, 3, 128), dtype=torch.bfloat16, device=DEV)
    rb.rtp_rope_append(d.ctx, d.params, d.cache()[1], rope, k, k, v, k_rot, None, tok_seq, tok_pos, d.status)
    check_rotated(k_rot, k, tok_pos, rope)
    b, plain = c.cache()
    rb.rtp_index_keys(c.ctx, c.params, plain, k[:, [2, 1]].contiguous(), w_k, tok_seq, tok_pos)
    rb.rtp_kv_append(c.ctx, c.params, plain, k_rot, v.contiguous(), tok_seq, tok_pos, c.status)
    assert c.code() == rb.RTP_OK
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_many_rows_take_the_same_values():
    """Enough rows for blocks of four passes; queries in place."""
    T = 2500
    c = Case([T], n_kv=4, group=8, n_ih=1)
    a, cache = c.cache()
    tok_seq, tok_pos = tokens([T], [T])
    q, k, v = rows(T, c, 1, fused=False)
    rope = rb.Rope(freqs(128))
    w_k = torch.randn((1, 128, 16), device=DEV).bfloat16()
    q0 = q.clone()
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, q, w_k, tok_seq, tok_pos, c.status)
    assert c.code() == rb.RTP_OK
    b, other = c.cache()
    out = torch.zeros_like(q)
    for lo in range(0, T, 100):   # a hundred tokens at a time: blocks of one pass
        s = slice(lo, min(T, lo + 100))
        rb.rtp_rope_append(c.ctx, c.params, other, rope, q0[s], k[s], v[s], out[s], w_k, tok_seq[s], tok_pos[s], c.status)
    assert torch.equal(q, out)
    for name in a:
        assert torch.equal(a[name], b[name]), name
    pick = [0, 1, 1249, 2499]
    check_rotated(q[pick], q0[pick], tok_pos[pick], rope)


def test_rows_that_cannot_be_written_are_skipped():
    c = Case([130, 130], refs=True)
    a, cache = c.cache()
    c.refs[int(c.table[1, 1])] = 2                     # a page that two sequences share
    c.table[0, 2] = -1
    tok_seq, tok_pos = i32([0, 1, 1, 0, 5, -1, 0, 0]), i32([3, 70, 3, 129, 3, 3, -1, 1 << 20])
    q, k, v = rows(8, c, 3)
    q_out = torch.zeros((8, c.n_q, 128), dtype=torch.bfloat16, device=DEV)
    w_k = torch.randn((1, 128, 16), device=DEV).bfloat16()
    rope = rb.Rope(freqs(128))
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, q_out, w_k, tok_seq, tok_pos, c.status)
    assert c.code() == rb.RTP_ERR_INVALID
    check_rotated(q_out, q, tok_pos, rope)
    written = {(int(c.table[0, 0]), 3), (int(c.table[1, 0]), 3)}
    for name in a:
        hit = (a[name].flatten(-1).float().abs().amax(-1).amax(1) > 0).nonzero().tolist()
        assert {tuple(x) for x in hit} == written, name


def test_nothing_to_do_and_refusals():
    c = Case([64])
    _, cache = c.cache()
    rope = rb.Rope(freqs(128))
    q, k, v = rows(3, c, 1)
    out = torch.zeros((3, c.n_q, 128), dtype=torch.bfloat16, device=DEV)
    s, p = i32([0, 0, 0]), i32([0, 1, 2])
    rb.rtp_rope_append(c.ctx, c.params, cache, rope, q[:0], k[:0], v[:0], out[:0], None, s[:0], p[:0], c.status)
    lib, h = c.ctx.lib, c.ctx.h
    import ctypes
    st = k.stride(0)

    def call(**o):
        a = dict(f=rope.freqs.data_ptr(), rd=128, il=0, sc=1.0, q=q.data_ptr(), qs=st, k=k.data_ptr(), ks=st, v=v.data_ptr(), vs=st,
                 out=out.data_ptr(), w=None, s=s.data_ptr(), p=p.data_ptr(), T=3)
        a.update(o)
        return lib.rtp_rope_append(h, c.params.ref(), ctypes.byref(cache), *a.values(), c.status.data_ptr(), None)

    assert call() == rb.RTP_OK
    for o in (dict(f=None), dict(k=None), dict(v=None), dict(s=None), dict(p=None), dict(q=None), dict(out=None), dict(rd=0), dict(rd=20), dict(rd=144),
              dict(sc=float("nan")), dict(sc=float("inf")), dict(q=q.data_ptr() + 2), dict(ks=4), dict(vs=st + 1), dict(qs=8), dict(T=-1),
              dict(q=out.data_ptr(), qs=st)):
        assert call(**o) == rb.RTP_ERR_INVALID, o
    assert call(T=1 << 31) == rb.RTP_ERR_UNSUPPORTED
    assert c.code() == rb.RTP_OK


def test_captured_and_replayed():
    c = Case([400, 400])
    a, cache = c.cache()
    tok_seq, tok_pos = tokens([10, 20], [4, 4])
    q, k, v = rows(8, c, 1)
    rope = rb.Rope(freqs(128))
    out = torch.zeros((8, c.n_q, 128), dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, out, None, tok_seq, tok_pos, c.status)
    for step in range(3):
        tok_pos += 64
        q.add_(step)
        g.replay()
        torch.cuda.synchronize()
        check_rotated(out, q, tok_pos, rope)
        at = (c.table[tok_seq.long(), tok_pos.long() // 64].long(), slice(None), tok_pos.long() % 64)
        check_rotated(a["k"][at], k, tok_pos, rope)
    assert c.code() == rb.RTP_OK
