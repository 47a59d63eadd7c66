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
