"""rtp_beam_select against 64 bits, and rtp_cache_reorder against its plain statement."""
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


def select(logits, scores, finished, beams, k, pad=3):
    ctx = rb.Context()
    rows, V = logits.shape
    G = rows // beams
    parent, token = (torch.full((G, k), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    out = torch.full((G, k), 9.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(rb.rtp_beam_workspace_bytes(rows, V, k), dtype=torch.uint8, device=DEV)
    rb.rtp_beam_select(ctx, logits, scores, finished, pad, parent, token, out, ws, status)
    return parent.cpu().numpy(), token.cpu().numpy(), out.cpu().numpy(), rb.rtp_check_status(ctx, status)


def check(logits, scores, finished, beams, k, pad=3):
    parent, token, out, code = select(logits, scores, finished, beams, k, pad)
    want = og.beam_select(logits.double().cpu().numpy(), None if scores is None else scores.double().cpu().numpy(),
                          None if finished is None else finished.cpu().numpy(), beams, k, pad)
    for g, w in enumerate(want):
        assert [(int(p), int(t)) for p, t in zip(parent[g], token[g])] == [(r, t) for _, r, t in w] + [(-1, -1)] * (k - len(w)), g
        for i, (s, _, _) in enumerate(w):
            # one rounding to 32 bits (2^-24 of the score) of a sum whose normaliser has a relative error below 2^-18 (a slice's 8192
            # terms of two ulp each summed in 32 bits: every partial sum of a thread, a warp and the slice rounds by 2^-24, 32 + 5 + 8 of them)
            assert (out[g, i] == s) if np.isinf(s) else abs(out[g, i] - s) <= 2.0 ** -24 * abs(s) + 2.0 ** -18, (g, i)
        assert (out[g, len(w):] == -np.inf).all()
    return code


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("G,W,V,k", [(1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 21), (1, 4, 2048, 8), (3, 2, 2049, 64), (2, 5, 4097, 33),
                                     (1, 64, 999, 64), (4, 8, 32000, 16), (40, 4, 50001, 9), (2, 64, 8190, 3)])
def test_sizes(G, W, V, k, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(V + k)
    x = (torch.randn((G * W, V), device=DEV, generator=g) * 3).to(dtype)
    s = -3 * torch.rand(G * W, device=DEV, generator=g)
    assert check(x, s, None, W, min(k, W * V)) == rb.RTP_OK


@pytest.mark.parametrize("V", [100, 8192, 40000])
def test_equal_logits_go_by_number(V):
    x = torch.zeros((6, V), device=DEV)
    assert check(x, None, None, 3, 40) == rb.RTP_OK
    x[:, V // 2:] = 1.0                                             # more equal ones than a list holds, not in front
    assert check(x, None, None, 3, 40) == rb.RTP_OK
    x[1] = x[4] = 0.0
    x[:, V - 20] = 2.0
    x[:, 17] = 2.0
    assert check(x.bfloat16(), None, None, 3, 64) == rb.RTP_OK


@pytest.mark.parametrize("V", [64, 3001, 20000])
def test_ruled_out_tokens_come_last(V):
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = torch.full((8, V), -torch.inf, device=DEV)
    x[0, V - 1] = 1.0                                               # one token
    x[2, ::7] = torch.randn(len(x[2, ::7]), device=DEV, generator=g)
    x[3, V // 2] = x[3, 3] = -3e38                                  # the type's lowest values are ordinary ones
    x[7, 5:9] = 2.0
    s = torch.tensor([0.0, 0, -1, -2, -torch.inf, -torch.inf, 0, -torch.inf], device=DEV)
    assert check(x, s, None, 4, 24) == rb.RTP_OK
    assert check(x, s, i32([0, 0, 0, 0, 0, 1, 0, 0]), 4, 24) == rb.RTP_OK


def test_ended_hypotheses_keep_their_score():
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x = torch.randn((12, 500), device=DEV, generator=g)
    s = -5 * torch.rand(12, device=DEV, generator=g)
    s[3] = 1.0
    assert check(x, s, i32([1, 0, 0, 1, 0, 1, 1, 1, 1, 1, 1, 1]), 4, 6, pad=499) == rb.RTP_OK   # (the last group: four continuations)
    assert check(x, s, i32([1] * 12), 4, 6, pad=-7) == rb.RTP_OK
    assert check(x[:1], s[:1], i32([1]), 1, 2) == rb.RTP_OK


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [50, 9001, 70000])
def test_zeros_of_either_sign_are_equal(V, dtype):
    x = torch.full((4, V), -0.0, device=DEV)
    x[:, 1::3] = 0.0
    x[2:, ::5] = -1.0
    x[:, V // 2:] *= -1.0
    x[1, V - 5:] = 2.0
    assert check(x.to(dtype), None, None, 2, 40) == rb.RTP_OK


def test_logits_that_rise_along_the_row():
    """Every group of chunks has more above the bound than a list holds."""
    V = 300000
    x = torch.arange(2 * V, device=DEV).remainder(V).reshape(2, V).float() / 1024
    assert check(x, None, None, 2, 64) == rb.RTP_OK
    x[1] = x[1].flip(0)
    assert check(x, None, None, 1, 3) == rb.RTP_OK


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [20000, 20003])
def test_large_logits_side_by_side_again_and_again(V, dtype):
    """Large logits at a fixed distance from each other, so that few threads have thousands of them, in rows that are not cut."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = torch.randn((600, V), device=DEV, generator=g)
    t = torch.arange(V, device=DEV)
    x[:, (t % 1024) < 300] += 50.0
    x[::2, (t % 2048) >= 1400] += 60.0
    assert check(x.to(dtype), None, None, 60, 64) == rb.RTP_OK


def test_peaked_rows_and_large_magnitudes():
    x = torch.zeros((4, 9000), device=DEV)
    x[0, 8999], x[1, 0], x[2] = 80.0, 1e4, -1e4
    x[3] = torch.linspace(-30, 30, 9000, device=DEV)
    assert check(x, None, None, 2, 17) == rb.RTP_OK
    x[3, 100:164] = torch.linspace(50, 40, 64, device=DEV)           # the best ones side by side, in one thread's hands
    assert check(x, None, None, 2, 64) == rb.RTP_OK


def test_what_is_no_number_is_reported():
    x = torch.randn((2, 3000), device=DEV)
    y = x.clone()
    x[0, 10], x[1, 2999] = torch.nan, torch.inf
    y[0, 10] = y[1, 2999] = -torch.inf
    got, want = select(x, None, None, 2, 9), select(y, None, None, 2, 9)
    assert got[3] == rb.RTP_ERR_INVALID and want[3] == rb.RTP_OK
    assert all((a == b).all() for a, b in zip(got[:3], want[:3]))
    s = torch.tensor([torch.nan, 0.0], device=DEV)
    parent, _, out, code = select(y, s, None, 2, 9)
    assert code == rb.RTP_ERR_INVALID and (parent == 1).all() and np.isfinite(out).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,stride", [(1001, 1003), (1000, 1001), (4096, 4104), (33, 1 << 12)])
def test_rows_with_strides(V, stride, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = torch.full((6, stride), 1e30, device=DEV, dtype=dtype)
    x[:, :V] = torch.randn((6, V), device=DEV, generator=g).to(dtype)
    assert check(x[:, :V], None, None, 3, 12) == rb.RTP_OK


def test_refusals():
    ctx = rb.Context()
    x = torch.zeros((4, 100), device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    o = torch.zeros(64, device=DEV)
    ws = torch.zeros(rb.rtp_beam_workspace_bytes(4, 100, 8), dtype=torch.uint8, device=DEV)

    def call(**over):
        a = dict(x=x.data_ptr(), f=rb.RTP_LOGITS_F32, rs=100, g=2, b=2, v=100, s=None, fin=None, pad=0, k=8, p=o.data_ptr(), t=o.data_ptr(), so=o.data_ptr(),
                 ws=ws.data_ptr(), n=ws.nbytes)
        a.update(over)
        return ctx.lib.rtp_beam_select(ctx.h, *a.values(), st.data_ptr(), None)

    assert call(g=0) == rb.RTP_OK
    for over in (dict(f=3), dict(rs=99), dict(b=0), dict(b=65), dict(k=0), dict(k=65), dict(v=0), dict(v=1 << 30), dict(g=-1), dict(x=None), dict(p=None),
                 dict(t=None), dict(so=None), dict(ws=None), dict(x=x.data_ptr() + 4), dict(b=1, v=7)):
        assert call(**over) == rb.RTP_ERR_INVALID, over
    assert call(n=ws.nbytes // 2) == rb.RTP_ERR_CAPACITY
    assert rb.rtp_beam_workspace_bytes(0, 100, 8) == rb.rtp_beam_workspace_bytes(4, 0, 8) == rb.rtp_beam_workspace_bytes(4, 100, 65) == 0


# ---- sequences that follow -------------------------------------------------------------------------------------------------
def moved(table, lens, refs, src, dst):
    ctx, params = rb.Context(), rb.Params(1, 1, [], [], [], [])
    k = torch.zeros((len(refs), 1, 64, 128), dtype=torch.bfloat16, device=DEV)
    t, ln, r = i32(table), i32(lens), i32(refs)
    cache = rb.make_cache(k, k, None, t, ln)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rb.rtp_cache_reorder(ctx, params, cache, r, i32(src), i32(dst), status)
    code = rb.rtp_check_status(ctx, status)
    wt, wl, wr, bad = og.reorder(table, lens, refs, src, dst)
    assert (t.cpu().numpy() == wt).all() and (ln.cpu().numpy() == wl).all() and (r.cpu().numpy() == wr).all()
    assert code == (rb.RTP_ERR_INVALID if bad else rb.RTP_OK)


def beams(B, cols, shared, seed):
    rng = np.random.default_rng(seed)
    own = cols - shared
    perm = rng.permutation(shared + B * own + 4)
    table = np.concatenate([np.tile(perm[:shared], (B, 1)), perm[shared:shared + B * own].reshape(B, own)], 1)
    for b in range(B):
        table[b, cols - rng.integers(0, own + 1):] = -1
    refs = np.zeros(len(perm), np.int64)
    np.add.at(refs, table[table >= 0], 1)
    return table, (table >= 0).sum(1) * 64 - 5, refs, rng


@pytest.mark.parametrize("B,cols,shared", [(1, 1, 0), (2, 3, 1), (8, 9, 5), (33, 130, 100), (300, 17, 3), (1500, 8, 2)])
def test_reorder(B, cols, shared):
    table, lens, refs, rng = beams(B, cols, shared, B)
    moved(table, lens, refs, rng.integers(0, B, B), np.arange(B))                 # a beam step
    moved(table, lens, refs, rng.permutation(B), rng.permutation(B))
    n = max(1, B // 2)
    moved(table, lens, refs, rng.integers(0, B, n), rng.permutation(B)[:n])        # some only
    moved(table, lens, refs, np.arange(B), np.arange(B))


def test_reorder_refuses_what_is_wrong():
    table, lens, refs, rng = beams(6, 5, 2, 7)
    moved(table, lens, refs, [0, 1, 2, 3], [3, 3, 2, 3])                          # named before
    moved(table, lens, refs, [0, -1, 6, 1], [1, 2, 3, -4])
    moved(table, lens, refs, [0, 1], [6, 2])
    table[4, 0] = len(refs) + 3                                                   # an entry that is no page is carried over
    moved(table, lens, refs, [4], [5])
    moved(table, lens, refs, list(range(6)) * 40, list(range(6)) * 40)


def test_a_reordered_pool_reserves_and_frees():
    """Hypotheses that share their last, partly filled page get copies of it."""
    from paper_2605_16928_b200 import pipeline
    params = rb.Params(2, 1, [], [], [], [])
    pool = pipeline.PagePool(params, 32, 4, 6)
    k = torch.randn((32, 1, 64, 128), device=DEV).bfloat16()
    v = torch.randn((32, 1, 64, 128), device=DEV).bfloat16()
    pool.cache_of(k, v)
    pool.reserve(i32([0]), i32([100]))
    pool.seq_lens[0] = 100
    pool.fork(i32([0, 0, 0]), i32([1, 2, 3]))
    pool.reserve(i32([0, 1, 2, 3]), i32([1, 1, 1, 1]))
    pool.seq_lens += 1
    assert pool.status_code() == rb.RTP_OK and int((pool.page_refs > 0).sum()) == 5
    pool.reorder(i32([2, 2, 2, 0]), i32([0, 1, 2, 3]))
    assert int((pool.page_refs > 0).sum()) == 3 and sorted(pool.page_refs[pool.page_refs > 0].tolist()) == [1, 3, 4]
    want = [k[pool.block_table[b, :2].long(), 0].reshape(-1, 128)[:101].clone() for b in range(4)]
    pool.reserve(i32([0, 1, 2, 3]), i32([1, 1, 1, 1]))
    assert pool.status_code() == rb.RTP_OK and int((pool.page_refs > 0).sum()) == 5
    for b in range(4):
        assert torch.equal(k[pool.block_table[b, :2].long(), 0].reshape(-1, 128)[:101], want[b])
    pool.free(i32([0, 1, 2, 3]))
    assert pool.status_code() == rb.RTP_OK and int(pool.page_refs.abs().sum()) == 0
