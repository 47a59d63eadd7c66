"""The 4-bit K/V cache on the GPU, through the C ABI, against the fp64 oracle: append and expansion bit for bit, decode
attention over every kind of set within the bounds that kv4_harness derives."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as k4
from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import synth

pytestmark = pytest.mark.gpu


def _h():
    from tests import kv4_harness
    return kv4_harness


def _special_values(rng, T, n_kv):
    """Rows of every size: normal ones, ties of every scale, zeros, the range's two ends."""
    x = rng.standard_normal((T, n_kv, 128)).astype(np.float32)
    for t in range(T):
        kind = t % 8
        if kind == 1:
            x[t] *= 2.0 ** -16
        elif kind == 2:
            x[t] = 0.0
        elif kind == 3:                      # exact ties: tie of the code times a scale, the group's maximum fixes the scale
            s = k4.SCALES[rng.integers(8, 220, (n_kv, 8, 1))]
            tie = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], (n_kv, 8, 16)) * rng.choice([-1, 1], (n_kv, 8, 16))
            tie[..., 0] = 6.0
            x[t] = (tie * s).reshape(n_kv, 128)
        elif kind == 4:
            x[t] *= 10000.0
        elif kind == 5:
            x[t] *= 2.0 ** rng.integers(-30, 12, (n_kv, 1))
        elif kind == 6:                      # maxima at ties of the scale
            x[t] = 0.0
            s = k4.SCALES[:219]
            i = rng.integers(0, 218, (n_kv, 8))
            x[t].reshape(n_kv, 8, 16)[..., 3] = 3.0 * (s[i] + s[i + 1])
    return synth.from_bf16(synth.to_bf16(x))


@pytest.mark.parametrize("T,n_kv,B", [(1, 1, 1), (65, 2, 1), (200, 8, 3), (1000, 4, 2)])
def test_append_is_bit_exact(T, n_kv, B):
    h = _h()
    rng = np.random.default_rng(T)
    c = h.Cache4([T] * B, n_kv=n_kv, group=1, ret_kv=())
    x, y = (_special_values(rng, B * T, n_kv) for _ in range(2))
    order = rng.permutation(B * T)
    seq, pos = (order // T).astype(np.int32), (order % T).astype(np.int32)
    before = [t.clone() for t in (c.d_k, c.d_v, c.d_s)]
    rb.rtp_kv_append(c.ctx, c.params, c.cache, h.dev_bf16(x), h.dev_bf16(y), h.dev_i32(seq), h.dev_i32(pos), c.status)
    assert c.code() == rb.RTP_OK
    got = [t.cpu().numpy() for t in (c.d_k, c.d_v, c.d_s)]
    ck, sk = k4.encode(x.astype(np.float64))
    cv, sv = k4.encode(y.astype(np.float64))
    used = np.zeros(c.kc.shape[:3], bool)
    for i in range(B * T):
        p, o = c.bt[seq[i], pos[i] // 64], pos[i] % 64
        used[p, :, o] = True
        assert np.array_equal(got[2][p, :, o], np.concatenate([sk[i], sv[i]], -1)), i
        # (the sign of a code that stands for zero is free)
        for a, b in ((k4.unpack(got[0][p, :, o]), ck[i]), (k4.unpack(got[1][p, :, o]), cv[i])):
            assert np.array_equal(np.where(a == 8, 0, a), np.where(b == 8, 0, b)), i
    for a, b in zip(got, before):
        assert np.array_equal(a[~used], b.cpu().numpy()[~used])


def test_append_reports_what_does_not_fit():
    h = _h()
    for bad in (np.nan, np.inf, -np.inf, 61696.0):
        c = h.Cache4([70], n_kv=2, group=1, ret_kv=())
        x = np.ones((3, 2, 128), np.float32)
        x[1, 1, 5] = bad
        rb.rtp_kv_append(c.ctx, c.params, c.cache, h.dev_bf16(x), h.dev_bf16(np.ones_like(x)), h.dev_i32([0] * 3), h.dev_i32([3, 4, 69]), c.status)
        assert c.code() == rb.RTP_ERR_UNSUPPORTED
        p = c.bt[0, 0]
        want = k4.encode(synth.from_bf16(synth.to_bf16(x[1, 1])).astype(np.float64))
        got = c.d_k[p, 1, 4].cpu().numpy(), c.d_s[p, 1, 4, :8].cpu().numpy()
        assert np.array_equal(k4.decode(k4.unpack(got[0]), got[1]), k4.decode(*want))
    c = h.Cache4([70], n_kv=2, group=1, ret_kv=())
    before = c.d_k.clone()
    rb.rtp_kv_append(c.ctx, c.params, c.cache, h.dev_bf16(x), h.dev_bf16(x), h.dev_i32([0, 1, -1]), h.dev_i32([128, 0, 0]), c.status)
    assert c.code() == rb.RTP_ERR_INVALID and torch.equal(before, c.d_k)


def test_expand_is_exact():
    h = _h()
    c = h.Cache4([130, 64, 1], n_kv=3, group=1, ret_kv=(), seed=4)
    src = np.concatenate([c.bt[0, :3], c.bt[1, :1], c.bt[2, :1]])
    dst = np.array([6, 0, 3, 2, 5])
    k = torch.full((8, 3, 64, 128), -77.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, -77.0)
    rb.rtp_kv_expand(c.ctx, c.params, c.cache, h.dev_i32(src), h.dev_i32(dst), k, v, c.status)
    assert c.code() == rb.RTP_OK
    for seq, rows in ((0, [(6, 64), (0, 64), (3, 2)]), (1, [(2, 64)]), (2, [(5, 1)])):
        for name, t in (("k", k), ("v", v)):
            got = torch.cat([t[p, :, :n].transpose(0, 1) for p, n in rows]).double().cpu().numpy()
            assert np.array_equal(got, getattr(c, name)[seq])
    assert (k[[1, 4, 7]] == -77).all() and (v[[1, 4, 7]] == -77).all()
    k2 = torch.zeros((5, 3, 64, 128), dtype=torch.bfloat16, device="cuda")
    rb.rtp_kv_expand(c.ctx, c.params, c.cache, h.dev_i32(src), None, k2, k2.clone(), c.status)
    assert torch.equal(k2[1].view(torch.int16), k[0].view(torch.int16)) and c.code() == rb.RTP_OK
    k3 = torch.full_like(k2, -77.0)
    rb.rtp_kv_expand(c.ctx, c.params, c.cache, h.dev_i32([c.kc.shape[0], -1, src[0], src[0], src[0]]), h.dev_i32([0, 1, 5, -1, 4]), k3,
                     k3.clone(), c.status)
    assert c.code() == rb.RTP_ERR_INVALID and (k3[:4] == -77).all() and torch.equal(k3[4].view(torch.int16), k[6].view(torch.int16))


@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 63, 64, 65, 130, 1000])
def test_dense_lengths_and_groups(L, group):
    c = _h().Cache4([L, max(1, L - 7)], n_kv=2, group=group, seed=L)
    rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check(range(c.n_q), lambda r, h: range(c.row_pos[r] + 1))


def test_dense_named_heads_positions_and_splits():
    h = _h()
    c = h.Cache4([5000, 300, 4999], n_kv=3, group=4, seed=9)
    rng = np.random.default_rng(3)
    seqs = [0, 0, 2, 1, 0]
    pos = [4999, 17, 4990, 299, 2500]
    c.set_rows(rng.standard_normal((5, 12, 128)), seqs, pos)
    rb.rtp_dense_attn_decode(*c.args(), [2, 0], c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check([h for h in range(12) if h // 4 in (0, 2)], lambda r, h: range(pos[r] + 1))
    a, b = c.out.clone(), c.lse.clone()
    c.out.fill_(-77), c.lse.fill_(-77)
    small = torch.empty(5 * 2 * 4 * 130 * 4 * 2 + 100, dtype=torch.uint8, device="cuda")     # room for two splits
    rb.rtp_dense_attn_decode(*c.args(), [2, 0], c.out, c.lse, small, c.status)
    c.check([h for h in range(12) if h // 4 in (0, 2)], lambda r, h: range(pos[r] + 1))
    one = torch.empty(16, dtype=torch.uint8, device="cuda")
    rb.rtp_dense_attn_decode(*c.args(), [2, 0], c.out, None, one, c.status)
    c.check([h for h in range(12) if h // 4 in (0, 2)], lambda r, h: range(pos[r] + 1))
    rb.rtp_dense_attn_decode(*c.args(), [2, 0], c.out, c.lse, c.ws, c.status)
    assert torch.equal(a, c.out) and torch.equal(b, c.lse)       # the same call, the same bits


def test_long_contexts_in_many_splits():
    """The results of all splits, of as many as the workspace has room for, and of a single one."""
    h = _h()
    L = 20000
    rng = np.random.default_rng(0)
    k, v = (np.tile(rng.standard_normal((500, 1, 128)), (40, 1, 1)) for _ in range(2))
    c = h.Cache4([L], n_kv=1, group=4, k=[k], v=[v], seed=9)
    full = rb.rtp_workspace_bytes(c.params, 1, L)
    for room in (full, 4 * 130 * 4 * 33, 4 * 130 * 4 * 17 + 5, 16):
        ws = torch.empty(room, dtype=torch.uint8, device="cuda")
        c.out.fill_(-77), c.lse.fill_(-77)
        rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, ws, c.status)
        c.check(range(4), lambda r, hd: range(L))
    idx = rng.permutation(L)[:9001]
    d_idx, d_cnt = h.dev_i32(np.tile(idx, (1, 4, 1))), h.dev_i32([[9001, 9000, 1, 0]])
    sets = lambda r, hd: idx[:[9001, 9000, 1, 0][hd]]
    for call in (rb.rtp_sparse_attn_decode, None):
        c.out.fill_(-77), c.lse.fill_(-77)
        if call:
            call(*c.args(), d_idx, d_cnt, c.out, c.lse, c.ws, c.status)
        else:
            rb.rtp_sparse_attn_decode_static(*c.args(), d_idx, d_cnt, c.out, c.lse, c.status)
        c.check(range(4), sets)
    assert c.code() == rb.RTP_OK


def test_static_scratch_takes_any_number_of_rows():
    """Where the built-in scratch would not hold the splits of a call, a 4-bit cache is read in fewer."""
    h = _h()
    c = h.Cache4([9000], n_kv=1, group=1, k=[np.tile(np.random.default_rng(1).standard_normal((300, 1, 128)), (30, 1, 1))])
    R = 700
    c.set_rows(np.random.default_rng(2).standard_normal((R, 1, 128)), [0] * R, [8999] * R)
    idx = np.stack([np.random.default_rng(r).permutation(9000)[:8500] for r in range(R)])[:, None]
    rb.rtp_sparse_attn_decode_static(*c.args(), h.dev_i32(idx), h.dev_i32(np.full((R, 1), 8500)), c.out, c.lse, c.status)
    assert c.code() == rb.RTP_OK
    c.check([0], lambda r, hd: idx[r, 0], rows=[0, 33, 699])


@pytest.mark.parametrize("scale", [1e-30, 1e-4, 1.0, 300.0, 1e20])
def test_query_magnitudes(scale):
    """Queries of any bf16 magnitude: they are scaled by a power of two on their way to fp16."""
    h = _h()
    c = h.Cache4([200], n_kv=1, group=4, seed=5, sm_scale=min(1.0, 1.0 / scale) * 128 ** -0.5)
    q = np.random.default_rng(0).standard_normal((1, 4, 128)) * scale
    q[0, 1] = 0.0
    q[0, 2, 1:] *= 1e-6
    c.set_rows(q, [0], [199])
    rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status)
    c.check(range(4), lambda r, h: range(200))


def test_rising_and_falling_scores():
    """The softmax reference trails the maximum: scores that climb by a little, by a lot and that fall off from the first."""
    h = _h()
    for slope in (0.05, 0.5, 40.0, -0.05, -3.0):
        n = 700
        k = np.zeros((n, 1, 128))
        k[:, 0, 0] = np.arange(n) * slope / 10.0
        c = h.Cache4([n], n_kv=1, group=2, k=[k], seed=1, sm_scale=1.0)
        q = np.zeros((1, 2, 128))
        q[0, :, 0] = [1.0, -1.0]
        c.set_rows(q, [0], [n - 1])
        rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status)
        c.check(range(2), lambda r, h: range(n))


@pytest.mark.parametrize("L,window,n_sink", [(1, 1, 0), (40, 5, 3), (100, 100, 4), (1000, 64, 4), (1000, 1, 70), (3000, 517, 17), (300, 4096, 4), (65, 64, 0)])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_local(L, window, n_sink, group):
    c = _h().Cache4([L, max(1, L // 2)], n_kv=3, group=group, ret_kv=(0,), local_kv=(2, 1), window=window, n_sink=n_sink, seed=L)
    rb.rtp_local_attn(*c.args(), 0, 0, c.R, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check([h for h in range(c.n_q) if h // group in (1, 2)],
            lambda r, h: [t for t in range(c.row_pos[r] + 1) if t < n_sink or t > c.row_pos[r] - window])


def _lists(c, rng, sizes, stride):
    n_ret = len(c.ret)
    idx = np.full((c.R, n_ret, stride), 1 << 30, np.int32)
    cnt = np.zeros((c.R, n_ret), np.int32)
    for r in range(c.R):
        for i in range(n_ret):
            n = min(sizes[(r * n_ret + i) % len(sizes)], int(c.row_pos[r]) + 1)
            idx[r, i, :n] = rng.permutation(int(c.row_pos[r]) + 1)[:n]
            cnt[r, i] = n
    return idx, cnt


@pytest.mark.parametrize("group", [1, 3, 4])
def test_lists(group):
    h = _h()
    c = h.Cache4([3000, 700, 1], n_kv=2, group=group, ret_kv=(1,), seed=2)
    idx, cnt = _lists(c, np.random.default_rng(0), [0, 1, 5, 16, 17, 2500, 64, 333], 2600)
    d_idx, d_cnt = h.dev_i32(idx), h.dev_i32(cnt)
    rb.rtp_sparse_attn_decode(*c.args(), d_idx, d_cnt, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    sets = lambda r, h: idx[r, c.ret.index(h), :cnt[r, c.ret.index(h)]]
    c.check(c.ret, sets)
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_sparse_attn_decode_static(*c.args(), d_idx, d_cnt, c.out, c.lse, c.status)
    c.check(c.ret, sets)
    # a token listed twice counts twice; counts beyond the stride are cut
    idx[0, 0, :4] = [5, 5, 5, 9]
    cnt[0, 0] = 4
    cnt[1, 0] = 9999
    n = min(700, 2600)
    idx[1, 0, :n] = np.random.default_rng(1).permutation(700)
    idx[1, 0, n:] = 3
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_sparse_attn_decode(*c.args(), h.dev_i32(idx), h.dev_i32(cnt), c.out, c.lse, c.ws, c.status)
    cnt[1, 0] = 2600
    c.check(c.ret, sets)
    assert c.code() == rb.RTP_OK


def test_lists_of_a_chunk():
    """The list form of the prefill call: rows are positions of one sequence."""
    h = _h()
    c = h.Cache4([400], n_kv=1, group=2, seed=8)
    C, q0 = 37, 300
    c.set_rows(np.random.default_rng(1).standard_normal((C, 2, 128)), [0] * C, q0 + np.arange(C))
    idx, cnt = _lists(c, np.random.default_rng(2), [1, 50, 200], 256)
    rb.rtp_sparse_attn_prefill(c.ctx, c.params, c.cache, c.d_q, None, None, 0, q0, C, h.dev_i32(idx), h.dev_i32(cnt), None, None, c.out,
                               c.lse, c.ws, c.status)
    c.check(c.ret, lambda r, h: idx[r, h, :cnt[r, h]])
    assert c.code() == rb.RTP_OK


def test_bad_entries_are_reported_and_skipped():
    h = _h()
    c = h.Cache4([100], n_kv=1, group=1, seed=3)
    idx = np.array([[[3, 100, 50, 7, 1 << 20, 99]]])
    rb.rtp_sparse_attn_decode(*c.args(), h.dev_i32(idx), h.dev_i32([[6]]), c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_ERR_INVALID
    c.check([0], lambda r, h: [3, 50, 7, 99])
    # rows without a sequence, and rows beyond theirs: reported; an empty set gives zeros and -inf
    c = h.Cache4([100, 64], n_kv=1, group=2, seed=3)
    c.set_rows(np.ones((4, 2, 128)), [-1, 1, 2, 0], [5, 70, 0, 30])
    rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_ERR_INVALID
    c.check(range(2), lambda r, h: [[], range(64), [], range(31)][r])


@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_pages(group):
    h = _h()
    c = h.Cache4([2000, 129, 64], n_kv=2, group=group, ret_kv=(0, 1), seed=group)
    rng = np.random.default_rng(group)
    n_ret = len(c.ret)
    idx = np.full((c.R, n_ret, 40), 1 << 20, np.int32)
    cnt = np.zeros((c.R, n_ret), np.int32)
    for r in range(c.R):
        n_pages = -(-c.lens[r] // 64)
        for i in range(n_ret):
            n = int(rng.integers(0, n_pages + 1))
            idx[r, i, :n] = rng.permutation(n_pages)[:n]
            cnt[r, i] = n
    sets = lambda r, h: [t for p in idx[r, c.ret.index(h), :cnt[r, c.ret.index(h)]] for t in range(64 * p, min(64 * p + 64, c.lens[r]))]
    d_idx, d_cnt = h.dev_i32(idx), h.dev_i32(cnt)
    rb.rtp_sparse_attn_decode_blocks(*c.args(), d_idx, d_cnt, c.out, c.lse, c.ws, c.status)      # grouped over the union
    assert c.code() == rb.RTP_OK
    c.check(c.ret, sets)
    c.out.fill_(-77), c.lse.fill_(-77)
    tiny = torch.empty(16, dtype=torch.uint8, device="cuda")                                    # every head for itself
    rb.rtp_sparse_attn_decode_blocks(*c.args(), d_idx, d_cnt, c.out, c.lse, tiny, c.status)
    assert c.code() == rb.RTP_OK
    c.check(c.ret, sets)


@pytest.mark.parametrize("group", [2, 4, 8])
def test_mixed_group(group):
    """A KV head with retrieval and local query heads: each call writes its own heads and leaves the others."""
    h = _h()
    c = h.Cache4([900, 70], n_kv=2, group=group, seed=group)
    ret = [0] if group == 2 else [0, 2]
    c.params = rb.Params(c.n_q, 2, ret, [0] * len(ret), [0], [0, 1], window=100, n_sink=3)
    c.ret = ret
    rb.rtp_local_attn(*c.args(), 0, 0, 2, c.out, c.lse, c.ws, c.status)
    local = lambda r, hd: [t for t in range(c.lens[r]) if t < 3 or t >= c.lens[r] - 100]
    c.check([hd for hd in range(c.n_q) if hd not in ret], local)
    c.out.fill_(-77), c.lse.fill_(-77)
    pages = [np.array([3, 0, 14, 7]), np.array([1])]
    idx = np.zeros((2, len(ret), 15), np.int32)
    for r in range(2):
        for i in range(len(ret)):
            idx[r, i, :len(pages[r]) - i * (r == 0)] = pages[r][:len(pages[r]) - i * (r == 0)]
    cnt = [[4 - i for i in range(len(ret))], [1] * len(ret)]
    sets = lambda r, hd: [t for p in idx[r, ret.index(hd), :cnt[r][ret.index(hd)]] for t in range(64 * p, min(64 * p + 64, c.lens[r]))]
    rb.rtp_sparse_attn_decode_blocks(*c.args(), h.dev_i32(idx), h.dev_i32(cnt), c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check(ret, sets)


def test_truncated_local_pool():
    """The local heads' own pool in 4 bits: the ring wraps; the results are those of the untruncated cache, bit for bit."""
    h = _h()
    L, window, n_sink = 1500, 256, 4
    rng = np.random.default_rng(0)
    k, v = (rng.standard_normal((L, 2, 128)) for _ in range(2))
    c = h.Cache4([L], n_kv=2, group=2, ret_kv=(0,), local_kv=(1,), window=window, n_sink=n_sink, k=[k], v=[v])
    rb.rtp_local_attn(*c.args(), 0, 0, 1, c.out, c.lse, c.ws, c.status)
    ref = c.out.clone(), c.lse.clone()
    c.check([2, 3], lambda r, h: [t for t in range(L) if t < n_sink or t > L - 1 - window])
    ring = window // 64 + 2
    slots = 1 + ring
    km, vm = (torch.full((c.kc.shape[0], 1, 64, 64), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    sm = torch.full((c.kc.shape[0], 1, 64, 16), 255, dtype=torch.uint8, device="cuda")
    kl, vl = (torch.full((slots + 2, 1, 64, 64), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    sl = torch.full((slots + 2, 1, 64, 16), 255, dtype=torch.uint8, device="cuda")
    lt = h.dev_i32(rng.permutation(slots + 2)[:slots][None])
    cache = rb.make_cache(km, vm, None, c.d_bt, c.d_lens, kl, vl, lt, 1, kv_scales=sm, kv_local_scales=sl)
    for lo in range(0, L, 200):
        hi = min(L, lo + 200)
        rb.rtp_kv_append(c.ctx, c.params, cache, h.dev_bf16(k[lo:hi]), h.dev_bf16(v[lo:hi]), h.dev_i32([0] * (hi - lo)), h.dev_i32(range(lo, hi)), c.status)
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_local_attn(c.ctx, c.params, cache, *c.args()[3:], 0, 0, 1, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    assert torch.equal(c.out, ref[0]) and torch.equal(c.lse, ref[1])
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_dense_attn_decode(c.ctx, c.params, cache, *c.args()[3:], [0], c.out, c.lse, c.ws, c.status)   # main pool: head 0
    assert c.code() == rb.RTP_OK
    c.check([0, 1], lambda r, h: range(L))


def test_another_stream_and_a_captured_graph():
    h = _h()
    c = h.Cache4([900, 333], n_kv=2, group=4, ret_kv=(0,), local_kv=(1,), window=100, seed=6)
    rng = np.random.default_rng(5)
    x, y = (rng.standard_normal((2, 2, 128)).astype(np.float32) for _ in range(2))
    dx, dy, seq, pos = h.dev_bf16(x), h.dev_bf16(y), h.dev_i32([0, 1]), h.dev_i32([899, 332])
    idx, cnt = _lists(c, rng, [300, 40, 7], 320)
    d_idx, d_cnt = h.dev_i32(idx), h.dev_i32(cnt)

    def step(stream=None):
        rb.rtp_kv_append(c.ctx, c.params, c.cache, dx, dy, seq, pos, c.status, stream=stream)
        rb.rtp_sparse_attn_decode(*c.args(), d_idx, d_cnt, c.out, c.lse, c.ws, c.status, stream=stream)
        rb.rtp_local_attn(*c.args(), 0, 0, 2, c.out, c.lse, c.ws, c.status, stream=stream)

    step()
    torch.cuda.synchronize()
    ref = c.out.clone(), c.lse.clone()
    for b, n in ((0, 899), (1, 332)):
        c.k[b][n], c.v[b][n] = (k4.decode(*k4.encode(synth.from_bf16(synth.to_bf16(z[b])).astype(np.float64))) for z in (x, y))
    sets = lambda r, h: idx[r, h, :cnt[r, h]] if h < 4 else [t for t in range(c.lens[r]) if t < 4 or t >= c.lens[r] - 100]
    c.check(range(8), sets)
    side = torch.cuda.Stream()
    c.out.zero_(), c.lse.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert torch.equal(c.out, ref[0]) and torch.equal(c.lse, ref[1])
    graph = torch.cuda.CUDAGraph()
    c.out.zero_(), c.lse.zero_()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        c.out.zero_(), c.lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, ref[0]) and torch.equal(c.lse, ref[1])
    assert c.code() == rb.RTP_OK


def test_prompt_through_expanded_pages():
    """A chunk appended to the 4-bit cache, its sequence expanded, the tensor-core prefill run on the expanded pages; the
    newest row's decode over the 4-bit pages gives the same."""
    h = _h()
    rng = np.random.default_rng(11)
    L, C = 500, 130
    k, v = (rng.standard_normal((L, 2, 128)) for _ in range(2))
    c = h.Cache4([L], n_kv=2, group=4, ret_kv=(0,), local_kv=(1,), window=200, k=[k], v=[v])
    q = rng.standard_normal((C, 8, 128))
    c.set_rows(q, [0] * C, L - C + np.arange(C))
    n_p = -(-L // 64)
    kx, vx = (torch.zeros((n_p, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rb.rtp_kv_expand(c.ctx, c.params, c.cache, c.d_bt[0, :n_p].contiguous(), None, kx, vx, c.status)
    scratch = rb.make_cache(kx, vx, None, h.dev_i32(np.arange(n_p)[None]), c.d_lens)
    rb.rtp_dense_attn_prefill(c.ctx, c.params, scratch, c.d_q, 0, L - C, C, None, c.out, c.lse, c.status)
    assert c.code() == rb.RTP_OK
    pre = c.out.clone()
    rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check(range(8), lambda r, h: range(c.row_pos[r] + 1), rows=[0, 64, C - 1])
    assert (pre.float() - c.out.float()).abs().max() <= 2e-2


def test_offsets_beyond_32_bits():
    """A pool whose codes take more than 4 GB: append, attention, expansion and page copies at its far end."""
    h = _h()
    n_kv, N, L = 8, 140000, 200                                # 32 KB of K codes a page: 4.6 GB
    rng = np.random.default_rng(0)
    k, v = (rng.standard_normal((L, n_kv, 128)) for _ in range(2))
    c = h.Cache4([L], n_kv=n_kv, group=2, ret_kv=(7,), local_kv=(3,), window=90, k=[k], v=[v])
    kp, vp = (torch.empty((N, n_kv, 64, 64), dtype=torch.uint8, device="cuda") for _ in range(2))
    sp = torch.empty((N, n_kv, 64, 16), dtype=torch.uint8, device="cuda")
    table = h.dev_i32([[N - 1, N - 3, 5, N - 2]])
    cache = rb.make_cache(kp, vp, None, table, c.d_lens, kv_scales=sp)
    p = (c.ctx, c.params, cache)
    rb.rtp_kv_append(*p, h.dev_bf16(k), h.dev_bf16(v), h.dev_i32([0] * L), h.dev_i32(range(L)), c.status)
    rb.rtp_cache_copy_pages(*p, h.dev_i32([N - 1, 5]), h.dev_i32([7, N - 9]), c.status)
    for row in ([N - 1, N - 3, 5, N - 2], [7, N - 3, N - 9, N - 2]):
        table.copy_(h.dev_i32([row]))
        c.out.fill_(-77), c.lse.fill_(-77)
        rb.rtp_dense_attn_decode(*p, *c.args()[3:], None, c.out, c.lse, c.ws, c.status)
        c.check(range(16), lambda r, hd: range(L))
        idx = rng.permutation(L)[:77]
        rb.rtp_sparse_attn_decode(*p, *c.args()[3:], h.dev_i32(np.tile(idx, (1, 2, 1))), h.dev_i32([[77, 77]]), c.out, c.lse, c.ws, c.status)
        rb.rtp_local_attn(*p, *c.args()[3:], 0, 0, 1, c.out, c.lse, c.ws, c.status)
        c.check(range(16), lambda r, hd: idx if hd >= 14 else [t for t in range(L) if hd not in (6, 7) or t < 4 or t >= L - 90])
    kx, vx = (torch.zeros((4, n_kv, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rb.rtp_kv_expand(*p, table[0], None, kx, vx, c.status)
    got = vx.transpose(1, 2).reshape(256, n_kv, 128)[:L].double().cpu().numpy()
    assert np.array_equal(got, c.v[0]) and c.code() == rb.RTP_OK


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, over the same cache."""
    h = _h()
    c = h.Cache4([3000, 2500], n_kv=2, group=4, ret_kv=(0,), local_kv=(1,), window=1000, seed=12)
    idx, cnt = _lists(c, np.random.default_rng(0), [700, 900], 1000)
    d_idx, d_cnt = h.dev_i32(idx), h.dev_i32(cnt)
    other = torch.empty_like(c.ws)
    side = torch.cuda.Stream()
    sets = lambda r, hd: idx[r, hd, :cnt[r, hd]] if hd < 4 else [t for t in range(c.lens[r]) if t < 4 or t >= c.lens[r] - 1000]
    ref = None
    for _ in range(20):
        c.out.fill_(-77), c.lse.fill_(-77)
        side.wait_stream(torch.cuda.current_stream())
        rb.rtp_local_attn(*c.args(), 0, 0, 2, c.out, c.lse, other, c.status, stream=side)
        rb.rtp_sparse_attn_decode(*c.args(), d_idx, d_cnt, c.out, c.lse, c.ws, c.status)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        if ref is None:
            c.check(range(8), sets)
            ref = c.out.clone(), c.lse.clone()
        assert torch.equal(c.out, ref[0]) and torch.equal(c.lse, ref[1])


def test_refusals():
    h = _h()
    c = h.Cache4([200], n_kv=2, group=2, ret_kv=(0,), local_kv=(1,))

    def refused(code, f, *a):
        c.out.fill_(-77)
        with pytest.raises(rb.RtpError) as e:
            f(*a)
        assert e.value.code == code and str(e.value)
        torch.cuda.synchronize()
        assert (c.out == -77).all()

    p = (c.ctx, c.params, c.cache)
    mask = torch.zeros((4, 2, 4), dtype=torch.int32, device="cuda")
    f = torch.zeros((4, 2), device="cuda")
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_dense_attn_prefill, *p, c.d_q, 0, 0, 1, None, c.out, c.lse, c.status)
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_local_attn, *p, c.d_q, None, None, 0, 0, 1, c.out, c.lse, c.ws, c.status)
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_sparse_attn_prefill_blocks, *p, c.d_q, 0, 0, 1, mask, c.out, c.lse, c.status)
    ik = torch.zeros((c.kc.shape[0], 1, 64, 16), dtype=torch.bfloat16, device="cuda")
    with_ikey = rb.make_cache(c.d_k, c.d_v, ik, c.d_bt, c.d_lens, kv_scales=c.d_s)
    w = torch.zeros((2, 128, 16), dtype=torch.bfloat16, device="cuda")
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_sparse_attn_prefill, c.ctx, c.params, with_ikey, c.d_q, c.d_q, w, 0, 0, 1, None, None, f,
            mask, c.out, c.lse, c.ws, c.status)
    pages = h.dev_i32([0])
    o = torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16, device="cuda")
    plain = rb.make_cache(o, o, None, c.d_bt, c.d_lens)
    refused(rb.RTP_ERR_UNSUPPORTED, rb.rtp_kv_expand, c.ctx, c.params, plain, pages, None, o, o, c.status)
    refused(rb.RTP_ERR_INVALID, rb.rtp_kv_expand, *p, pages, None, o.view(-1)[1:].view(1, -1), o, c.status)
    for change in (dict(kv_format=7), dict(kv_scales=None), dict(kv_scales=c.d_s.data_ptr() + 4)):
        bad = rb.make_cache(c.d_k, c.d_v, None, c.d_bt, c.d_lens, kv_scales=c.d_s)
        for name, value in change.items():
            setattr(bad, name, value)
        refused(rb.RTP_ERR_INVALID, rb.rtp_dense_attn_decode, c.ctx, c.params, bad, *c.args()[3:], None, c.out, c.lse, c.ws, c.status)
    c3 = h.Cache4([20], n_kv=1, group=3)
    with pytest.raises(rb.RtpError) as e:
        rb.rtp_dense_attn_decode(*c3.args(), None, c3.out, c3.lse, c3.ws, c3.status)
    assert e.value.code == rb.RTP_ERR_UNSUPPORTED
