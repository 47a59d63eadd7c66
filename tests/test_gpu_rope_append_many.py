"""rtp_rope_append of thousands of tokens in all its forms: the same bits as a hundred tokens at a time, which the other tests hold against
64 bits, and a few rows against 64 bits here as well."""
import numpy as np
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_rope_append import DEV, Case, check_rotated, freqs, i32, rows, tokens

pytestmark = pytest.mark.gpu
T = 2403                                           # more than two blocks of eight tokens per SM, and not a whole number of them


def both(c, rope, with_q, n_ih, tok_seq, tok_pos, seed, fused=True):
    """One call, and calls of a hundred tokens: the arrays of both, the rotated queries, the statuses."""
    q, k, v = rows(len(tok_seq), c, seed, fused)
    w_k = torch.randn((n_ih, 128, 16), device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).bfloat16() if n_ih else None
    res = []
    for step in (len(tok_seq), 100):
        a, cache = c.cache()
        out = torch.full((len(tok_seq), c.n_q, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        for lo in range(0, len(tok_seq), step):
            s = slice(lo, min(len(tok_seq), lo + step))
            rb.rtp_rope_append(c.ctx, c.params, cache, rope, q[s] if with_q else None, k[s], v[s], out[s] if with_q else None, w_k, tok_seq[s], tok_pos[s], c.status)
        res.append((a, out, c.code()))
    for name in res[0][0]:
        assert torch.equal(res[0][0][name], res[1][0][name]), name
    assert torch.equal(res[0][1], res[1][1]) and res[0][2] == res[1][2]
    return res[0], q


@pytest.mark.parametrize("rd,interleaved,scale", [(128, True, 1.0), (64, False, 0.5), (96, True, -1.25), (16, False, 1.0), (48, False, 1.0), (128, False, 1.0)])
@pytest.mark.parametrize("with_q,n_ih,e4m3,fused", [(True, 2, False, True), (False, 1, True, True), (True, 0, False, False)])
def test_rotations(rd, interleaved, scale, with_q, n_ih, e4m3, fused):
    lens, new = [1300, 900, 400], [1203, 900, 300]
    c = Case(lens, n_kv=3, group=3, n_ih=n_ih, e4m3=e4m3, seed=rd)
    tok_seq, tok_pos = tokens(lens, new)
    rope = rb.Rope(freqs(rd), rd, interleaved, scale)
    (_, out, code), q = both(c, rope, with_q, n_ih, tok_seq, tok_pos, rd, fused)
    assert code == rb.RTP_OK and len(tok_seq) == T
    if with_q:
        pick = [0, 7, 8, 1203, 2399, T - 1]
        check_rotated(out[pick], q[pick], tok_pos[pick], rope)


@pytest.mark.parametrize("local", [(0,), (0, 2), (0, 1, 2)])
@pytest.mark.parametrize("fp4", [False, True])
def test_truncated_pools(local, fp4):
    lens = [300 - 7 * i for i in range(21)]        # (a ring of three pages takes 192 tokens of a sequence at a time)
    new = [114] * 20 + [T - 20 * 114]
    c = Case(lens, n_kv=3, group=2, n_ih=2, fp4=fp4, local=local, seed=len(local))
    tok_seq, tok_pos = tokens(lens, new)
    (_, out, code), q = both(c, rb.Rope(freqs(96, 500000.0), 96), True, 2, tok_seq, tok_pos, 5)
    assert code == rb.RTP_OK
    check_rotated(out[::400], q[::400], tok_pos[::400], rb.Rope(freqs(96, 500000.0), 96))


def test_rows_that_cannot_be_written_are_skipped():
    """Shared pages, unmapped ones, sequences and positions out of range, among thousands that are written; in no order."""
    c = Case([1300, 1300], refs=True, seed=9)
    c.refs[c.table[0, 3].long()] = 2
    c.refs[c.table[1, 0].long()] = 0
    c.table[1, 7], c.table[0, 5] = -1, 1 << 20
    order = torch.randperm(2600, generator=torch.Generator().manual_seed(1))[:T].to(DEV)
    tok_seq, tok_pos = (order // 1300).int(), (order % 1300).int()
    tok_seq[5::97], tok_seq[11::201], tok_pos[17::300], tok_pos[40::500] = -1, 2, -3, 1 << 30
    rope = rb.Rope(freqs(128))
    (a, out, code), q = both(c, rope, True, 1, tok_seq, tok_pos, 3)
    assert code == rb.RTP_ERR_INVALID
    check_rotated(out[::300], q[::300], tok_pos[::300], rope)            # (queries are rotated whatever becomes of the append)
    ok = (tok_seq >= 0) & (tok_seq < 2) & (tok_pos >= 0) & (tok_pos < 1300)
    page = torch.where(ok, c.table[tok_seq.clamp(0, 1).long(), tok_pos.clamp(0, 1299).long() // 64], -1)
    ok &= (page >= 0) & (page < c.N)
    ok &= torch.where(ok, c.refs[page.clamp(0, c.N - 1).long()], 0) == 1
    want = {(int(p), int(x) % 64) for p, x in zip(page[ok], tok_pos[ok])}
    assert {tuple(x) for x in (a["v"].float().abs().amax(-1).amax(1) > 0).nonzero().tolist()} == want and len(want) > 1500


def test_captured_with_queries_in_place():
    c = Case([5000], n_kv=2, group=4, n_ih=1, seed=2)
    tok_seq, tok_pos = tokens([2500], [T])
    q, k, v = rows(T, c, 2, fused=False)
    rope = rb.Rope(freqs(128))
    w_k = torch.randn((1, 128, 16), device=DEV).bfloat16()
    a, cache = c.cache()
    q0, side, g = q.clone(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        rb.rtp_rope_append(c.ctx, c.params, cache, rope, q, k, v, q, w_k, tok_seq, tok_pos, c.status)
    for _ in range(2):
        q.copy_(q0)
        tok_pos += 700
        g.replay()
        torch.cuda.synchronize()
        pick = [0, 1000, T - 1]
        check_rotated(q[pick], q0[pick], tok_pos[pick], rope)
        page = c.table[0, tok_pos[pick].long() // 64].long()
        check_rotated(a["k"][page, :, tok_pos[pick].long() % 64], k[pick], tok_pos[pick], rope)
    assert c.code() == rb.RTP_OK
