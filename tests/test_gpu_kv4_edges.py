"""Attention over a 4-bit cache where inputs are unusual: queries that are not numbers, wide and wrong tables, few listed heads."""
import numpy as np
import pytest
import torch

from paper_2605_16928_b200 import binding as rb

pytestmark = pytest.mark.gpu


def _h():
    from tests import kv4_harness
    return kv4_harness


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("L", [1, 40, 3000])
def test_a_query_that_is_not_a_number(L, group, bad):
    """Heads whose query holds a NaN or an infinity answer NaN (every product with it and a key of either sign, or zero, is in the
    sum); the other heads, and heads without a token, answer as ever.  One split and many, every kind of set."""
    h = _h()
    rng = np.random.default_rng(L)
    # (a NaN among infinities: a channel whose key is zero somewhere in the set)
    k = rng.standard_normal((L, 2, 128))
    k[0, :, 5] = 0.0
    c = h.Cache4([L], n_kv=2, group=group, ret_kv=(0,), local_kv=(1,), window=max(1, L), n_sink=1, seed=L, k=[k])
    q = rng.standard_normal((1, 2 * group, 128)).astype(np.float32)
    wrong = [0, 2 * group - 1]
    for x in wrong:
        q[0, x, 5] = bad
    c.set_rows(np.where(np.isfinite(q), q, 0.0), [0], [L - 1])
    c.d_q = torch.from_numpy(q).to("cuda").bfloat16()
    tok = h.dev_i32(np.tile(np.arange(L), (1, group, 1)))
    cnt = h.dev_i32(np.full((1, group), L))
    page = h.dev_i32(np.tile(np.arange(-(-L // 64)), (1, group, 1)))
    n_page = h.dev_i32(np.full((1, group), -(-L // 64)))
    small = torch.empty(16, dtype=torch.uint8, device="cuda")

    def answer(heads, call):
        c.out.fill_(-77), c.lse.fill_(-77)
        call()
        assert c.code() == rb.RTP_OK
        out, lse = c.out.clone(), c.lse.clone()
        out[:, wrong], lse[:, wrong] = -77, -77
        c.check([x for x in heads if x not in wrong], lambda r, hd: range(L), out=out, lse=lse)
        for x in wrong:
            if x in heads:
                assert torch.isnan(c.out[0, x]).all() and torch.isnan(c.lse[0, x]), (x, c.lse[0, x])
            else:
                assert (c.out[0, x] == -77).all()

    every, ret, loc = range(2 * group), range(group), range(group, 2 * group)
    for ws in (c.ws, small):
        answer(every, lambda: rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, ws, c.status))
        answer(loc, lambda: rb.rtp_local_attn(*c.args(), 0, 0, 1, c.out, c.lse, ws, c.status))
        answer(ret, lambda: rb.rtp_sparse_attn_decode(*c.args(), tok, cnt, c.out, c.lse, ws, c.status))
        answer(ret, lambda: rb.rtp_sparse_attn_decode_blocks(*c.args(), page, n_page, c.out, c.lse, ws, c.status))
    # nothing to attend to: zeros and -inf whatever the query
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_sparse_attn_decode(*c.args(), tok, torch.zeros_like(cnt), c.out, c.lse, c.ws, c.status)
    assert not c.out[0, :group].any() and (c.lse[0, :group] == -np.inf).all()


@pytest.mark.parametrize("ret", [[0], [7], [1, 6], [0, 3, 5], [0, 1, 2, 4, 7], list(range(8))])
def test_page_lists_of_some_heads_of_a_group(ret):
    """Any number of a group's eight heads with a list, lists of any length (none at all for one), pages of every word."""
    h = _h()
    L, W = 5000, 79
    c = h.Cache4([L, 700], n_kv=1, group=8, k=[np.tile(np.random.default_rng(0).standard_normal((100, 1, 128)), (n // 100, 1, 1)) for n in (L, 700)])
    c.params = rb.Params(8, 1, ret, [0] * len(ret), [0], [])
    c.ret = ret
    rng = np.random.default_rng(len(ret))
    cnt = np.array([[[W, 0, 40, 1, 79, 13, 3, 64][i] for i in range(len(ret))], [min(11, 1 + 3 * i) for i in range(len(ret))]])
    idx = np.stack([[rng.permutation(n)[np.arange(W) % n] for _ in ret] for n in (W, 11)])
    sets = lambda r, hd: [t for p in idx[r, ret.index(hd), :cnt[r, ret.index(hd)]] for t in range(64 * p, min(64 * p + 64, c.lens[r]))]
    rb.rtp_sparse_attn_decode_blocks(*c.args(), h.dev_i32(idx), h.dev_i32(cnt), c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK
    c.check(ret, sets)


@pytest.mark.parametrize("n_pages", [8191, 8193, 16384, 16400])
def test_page_lists_of_long_tables(n_pages):
    """Unions of up to 512 words of 32 pages and beyond: every listed page of a list without an order is attended to once per head
    (a table that maps all pages of a sequence to one: the log-sum-exp counts the tokens)."""
    h = _h()
    c = h.Cache4([64], n_kv=1, group=4, k=[np.zeros((64, 1, 128))])
    L = 64 * n_pages - 5
    table = h.dev_i32(np.full((1, n_pages), c.bt[0, 0]))
    lens = h.dev_i32([L])
    cache = rb.make_cache(c.d_k, c.d_v, None, table, lens, kv_scales=c.d_s)
    c.params = rb.Params(4, 1, [0, 2, 3], [0] * 3, [0], [])
    cnt = np.array([[n_pages, 1000, 1]])
    rng = np.random.default_rng(n_pages)
    idx = np.stack([rng.permutation(n_pages) for _ in range(3)])[None]
    idx[0, 2, 0] = n_pages - 1
    ws = torch.empty(rb.rtp_workspace_bytes(c.params, 1, L), dtype=torch.uint8, device="cuda")
    rb.rtp_sparse_attn_decode_blocks(c.ctx, c.params, cache, c.d_q, h.dev_i32([0]), h.dev_i32([L - 1]), h.dev_i32(idx), h.dev_i32(cnt),
                                     c.out, c.lse, ws, c.status)
    assert c.code() == rb.RTP_OK
    tokens = [64 * n - 5 * bool((idx[0, i, :n] == n_pages - 1).any()) for i, n in enumerate(cnt[0])]
    lse = c.lse[0, [0, 2, 3]].double().cpu().numpy()
    # scores are zero: sums of ones (times 2^7), exact in fp32 up to 2^24; a logarithm and a product in fp32
    assert (np.abs(lse - np.log(tokens)) <= 2.0 ** -22 * np.log(tokens)).all(), (lse, np.log(tokens))
    v = c.v[0][:, 0]
    want = v.mean(0)
    got = c.out[0, 0].double().cpu().numpy()
    # all heads but the tail of five tokens in one page: the mean moves by at most 5 |v| / L; fp16 probabilities are exact (2^7)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 20 * np.abs(v).max() / L + 2.0 ** -14).all()


def test_a_chunk_over_a_4bit_local_pool():
    """The chunk form is refused, without the advice to expand a pool that no call expands; the same rows as row arrays answer
    like the rows over one pool, bit for bit."""
    h = _h()
    L, C, window = 400, 50, 100
    rng = np.random.default_rng(3)
    k, v = (rng.standard_normal((L, 2, 128)) for _ in range(2))
    c = h.Cache4([L], n_kv=2, group=2, ret_kv=(0,), local_kv=(1,), window=window, n_sink=4, k=[k], v=[v])
    c.set_rows(rng.standard_normal((C, 4, 128)), [0] * C, L - C + np.arange(C))
    kl, vl = (torch.full((8, 1, 64, 64), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    sl = torch.full((8, 1, 64, 16), 255, dtype=torch.uint8, device="cuda")
    ring = 6
    km, vm, sm = (x[:, :1].contiguous() for x in (c.d_k, c.d_v, c.d_s))
    table = h.dev_i32(rng.permutation(8)[:1 + ring][None])
    cache = rb.make_cache(km, vm, None, c.d_bt, c.d_lens, kl, vl, table, 1, kv_scales=sm, kv_local_scales=sl)
    for lo in range(0, L, 100):
        rb.rtp_kv_append(c.ctx, c.params, cache, h.dev_bf16(k[lo:lo + 100]), h.dev_bf16(v[lo:lo + 100]), h.dev_i32([0] * 100),
                         h.dev_i32(range(lo, lo + 100)), c.status)
    p = (c.ctx, c.params, cache)
    with pytest.raises(rb.RtpError) as e:
        rb.rtp_local_attn(*p, c.d_q, None, None, 0, L - C, C, c.out, c.lse, c.ws, c.status)
    assert e.value.code == rb.RTP_ERR_UNSUPPORTED and "expand" not in str(e.value)
    rb.rtp_local_attn(*c.args(), 0, 0, C, c.out, c.lse, c.ws, c.status)
    want = c.out.clone(), c.lse.clone()
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_local_attn(*p, *c.args()[3:], 0, 0, C, c.out, c.lse, c.ws, c.status)
    assert c.code() == rb.RTP_OK and torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])
    c.check([2, 3], lambda r, hd: [t for t in range(c.row_pos[r] + 1) if t < 4 or t > c.row_pos[r] - window])


def test_launches_of_a_prefill_chunk_are_counted():
    from torch.profiler import ProfilerActivity, profile

    from paper_2605_16928_b200 import pipeline, synth_device
    L = 300
    data = synth_device.config_3_device(L=L, window=100)
    for kv_fp4 in (False, True):
        path = pipeline.PrefillPath(data, L, kv_fp4=kv_fp4)
        out = torch.zeros((L, 32, 128), dtype=torch.bfloat16, device="cuda")
        kp = data.k_pre_rows(0, 0, L)
        path.run_chunk(0, L, data.q[:L], kp, out)
        torch.cuda.synchronize()
        with profile(activities=[ProfilerActivity.CUDA]) as p:
            path.run_chunk(0, L, data.q[:L], kp, out)
            torch.cuda.synchronize()
        kernels = [e for e in p.events() if e.device_type == torch.autograd.DeviceType.CUDA and "rtp::" in e.name]
        assert len(kernels) == path.launches_per_chunk, [e.name for e in kernels]


@pytest.mark.parametrize("cols", [0, 70, 2048, 16384])
def test_tables_wider_than_their_sequences(cols):
    """A server's table is as wide as its longest context: splits are planned for that, the sequences are short."""
    h = _h()
    c = h.Cache4([4096, 1, 700], n_kv=2, group=4, ret_kv=(0,), local_kv=(1,), window=500, seed=7, table_cols=cols,
                 k=[np.tile(np.random.default_rng(b).standard_normal((min(n, 128), 2, 128)), (max(1, n // 128), 1, 1))[:n] if n != 700 else
                    np.random.default_rng(9).standard_normal((700, 2, 128)) for b, n in enumerate([4096, 1, 700])])
    ws = torch.empty(max(c.ws.numel(), rb.rtp_workspace_bytes(c.params, 3, 64 * max(64, cols))), dtype=torch.uint8, device="cuda")
    rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, ws, c.status)
    c.check(range(8), lambda r, hd: range(c.lens[r]))
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_local_attn(*c.args(), 0, 0, 3, c.out, c.lse, ws, c.status)
    c.check(range(4, 8), lambda r, hd: [t for t in range(c.lens[r]) if t < 4 or t >= c.lens[r] - 500])
    rng = np.random.default_rng(cols)
    n_pages = [-(-n // 64) for n in c.lens]
    cnt = np.array([[rng.integers(0, n + 1) for _ in range(4)] for n in n_pages])
    idx = np.stack([[rng.permutation(n)[np.arange(64) % n] for _ in range(4)] for n in n_pages])
    sets = lambda r, hd: [t for p in idx[r, hd, :cnt[r, hd]] for t in range(64 * p, min(64 * p + 64, c.lens[r]))]
    for w in (ws, torch.empty(16, dtype=torch.uint8, device="cuda")):
        c.out.fill_(-77), c.lse.fill_(-77)
        rb.rtp_sparse_attn_decode_blocks(*c.args(), h.dev_i32(idx), h.dev_i32(cnt), c.out, c.lse, w, c.status)
        c.check(range(4), sets)
    cnt = np.array([[min(n, 900), 1, 0, n // 2] for n in c.lens])
    idx = np.stack([[rng.permutation(n)[np.arange(900) % n] for _ in range(4)] for n in c.lens])
    c.out.fill_(-77), c.lse.fill_(-77)
    rb.rtp_sparse_attn_decode(*c.args(), h.dev_i32(idx), h.dev_i32(cnt), c.out, c.lse, ws, c.status)
    cnt = np.minimum(cnt, 900)
    c.check(range(4), lambda r, hd: idx[r, hd, :cnt[r, hd]])
    assert c.code() == rb.RTP_OK


@pytest.mark.parametrize("entry", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_table_entries_that_name_no_page(entry):
    """An unmapped entry inside a sequence, or one beyond the pool: reported; the rows of other sequences answer as ever."""
    h = _h()
    c = h.Cache4([300, 200], n_kv=2, group=2, ret_kv=(0,), local_kv=(1,), window=250, seed=3)
    c.d_bt[0, 2] = entry
    tok, cnt = h.dev_i32(np.tile(np.arange(200), (2, 2, 1))), h.dev_i32(np.full((2, 2), 200))
    page, n_page = h.dev_i32(np.tile(np.arange(4), (2, 2, 1))), h.dev_i32(np.full((2, 2), 4))
    local = lambda r, hd: [t for t in range(200) if t < 4 or t >= 200 - 250]
    for call, heads, sets in (
            (lambda: rb.rtp_dense_attn_decode(*c.args(), None, c.out, c.lse, c.ws, c.status), range(4), lambda r, hd: range(200)),
            (lambda: rb.rtp_local_attn(*c.args(), 0, 0, 2, c.out, c.lse, c.ws, c.status), range(2, 4), local),
            (lambda: rb.rtp_sparse_attn_decode(*c.args(), tok, cnt, c.out, c.lse, c.ws, c.status), range(2), lambda r, hd: range(200)),
            (lambda: rb.rtp_sparse_attn_decode_blocks(*c.args(), page, n_page, c.out, c.lse, c.ws, c.status), range(2), lambda r, hd: range(200))):
        c.status.zero_()
        c.out.fill_(-77), c.lse.fill_(-77)
        call()
        assert c.code() == rb.RTP_ERR_INVALID
        c.check(heads, sets, rows=[1])
