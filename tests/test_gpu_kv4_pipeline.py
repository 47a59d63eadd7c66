"""The decode and prefill paths on a 4-bit K/V cache against the same paths on the bf16 cache that holds its values: the same
selection, attention within the rounding of the two kernels (probabilities in fp16 here, in bf16 there)."""
import dataclasses

import pytest
import torch

from paper_2605_16928_b200 import binding as rb

pytestmark = pytest.mark.gpu

# Outputs are sums of p v with |v| <= 6 (N(0, 1) values): half a bf16 step of the result twice, and of every p once, give
# 2^-8 * (2 |o| + sum p |v|) <= 2^-8 * 3 * max |v|, about 0.07 at the most; the mean over the outputs (|o| and sum p |v| of
# order one) stays below 2^-8 * 3.
MAX_DIFF, MEAN_DIFF = 0.07, 3 * 2.0 ** -8


def _widened(data, path):
    """The workload with the values that the 4-bit cache holds in place of its own K/V rows."""
    ids = torch.arange(data.num_pages, dtype=torch.int32, device="cuda")
    k, v = torch.zeros_like(data.k_pages), torch.zeros_like(data.v_pages)
    rb.rtp_kv_expand(path.ctx, path.params, path.cache, ids, None, k, v, path.status)
    return dataclasses.replace(data, k_pages=k, v_pages=v)


def _close(a, b):
    d = (a.float() - b.float()).abs()
    assert d.max() <= MAX_DIFF and d.mean() <= MEAN_DIFF, (d.max(), d.mean())


@pytest.mark.parametrize("ikey_e4m3", [False, True])
def test_decode_steps(ikey_e4m3):
    from paper_2605_16928_b200 import pipeline, synth_device
    data = synth_device.decode_device(L=5000, batch=3, top_p=0.9, frac=0.1, window=700)
    a = pipeline.DecodePath(data, sel_stride=5000, kv_fp4=True, ikey_e4m3=ikey_e4m3)
    wide = _widened(data, a)
    b = pipeline.DecodePath(wide, sel_stride=5000, ikey_e4m3=ikey_e4m3)
    k_new = torch.stack([data.k_pages[data.block_table[s, 4999 // 64].long(), data.heads.index_head_kv, 4999 % 64] for s in range(3)])
    for path in (a, b):
        path.build_index_cache()     # (from the workload's own keys, quantised or not: let both score the same)
    a.ikey_pages.copy_(b.ikey_pages)
    k_new = k_new.contiguous()
    for step in ("step", "step_blocks"):
        for path in (a, b):
            path.out.zero_()
            getattr(path, step)(data.q, k_new)
        torch.cuda.synchronize()
        assert a.status_code() == rb.RTP_OK and b.status_code() == rb.RTP_OK
        if step == "step":
            assert torch.equal(a.sel_cnt, b.sel_cnt)
        _close(a.out, b.out)
        assert (a.lse - b.lse).abs().max() <= 1e-3
    for path in (a, b):
        path.step_dense(data.q)
    _close(a.out, b.out)


def test_prefill_chunks():
    from paper_2605_16928_b200 import pipeline, synth_device
    L, C = 1500, 512
    data = synth_device.config_3_device(L=L, window=300)
    a = pipeline.PrefillPath(data, C, kv_fp4=True)
    b = pipeline.PrefillPath(_widened(data, a), C)
    outs = []
    for path in (a, b):
        out = torch.zeros((L, 32, 128), dtype=torch.bfloat16, device="cuda")
        blocks, dense = torch.zeros_like(out), torch.zeros_like(out)
        for lo, n in path.chunks():
            kp = data.k_pre_rows(0, lo, lo + n)
            path.run_chunk(lo, n, data.q[lo:lo + n], kp, out[lo:lo + n])
            path.run_chunk_blocks(lo, n, data.q[lo:lo + n], kp, blocks[lo:lo + n])
            path.run_chunk_dense(lo, n, data.q[lo:lo + n], dense[lo:lo + n])
        torch.cuda.synchronize()
        assert path.status_code() == rb.RTP_OK
        outs.append((out, blocks, dense))
    for x, y in zip(*outs):           # the same kernels on the same values
        assert torch.equal(x, y)


def test_page_pool():
    """Two prompts come, one is forked, one leaves, the pool is compacted; lengths and tables as the calls promise."""
    from paper_2605_16928_b200 import pipeline
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    params = rb.Params(2, 1, [], [], [], [])
    pool = pipeline.PagePool(params, num_pages=16, batch=4, max_pages=6)
    k, v = (torch.zeros((16, 1, 64, 64), dtype=torch.uint8, device="cuda") for _ in range(2))
    scales = torch.zeros((16, 1, 64, 16), dtype=torch.uint8, device="cuda")
    cache = pool.cache_of(k, v, kv_scales=scales)
    pool.reserve(i32(0, 1), i32(130, 100))
    rows = torch.randn((230, 1, 128), device="cuda").bfloat16()
    seq = torch.cat([torch.zeros(130), torch.ones(100)]).int().cuda()
    pos = torch.cat([torch.arange(130), torch.arange(100)]).int().cuda()
    rb.rtp_kv_append(pool.ctx, params, cache, rows, -rows, seq, pos, pool.status)
    pool.seq_lens[:2] = i32(130, 100)
    pool.fork(i32(1), i32(2))
    pool.reserve(i32(2), i32(1))
    assert pool.block_table[2].tolist() == [3, 5, -1, -1, -1, -1] and pool.page_refs[:6].tolist() == [1, 1, 1, 2, 1, 1]
    pool.free(i32(0))
    pool.compact()
    assert int(pool.n_used) == 3 and pool.block_table[1].tolist()[:2] == [0, 1] and pool.block_table[2].tolist()[:2] == [0, 2]
    assert torch.equal(k[1], k[2]) and k[1].any() and torch.equal(scales[1], scales[2])
    pool.reserve(i32(3), i32(64 * 14))
    assert pool.status_code() == rb.RTP_ERR_CAPACITY and int((pool.page_refs > 0).sum()) == 3
