"""What the binding itself refuses: descriptions that the library, which sees pointers only, cannot check."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb


def _cache(**over):
    k, v = (torch.zeros((6, 2, 64, 64), dtype=torch.uint8) for _ in range(2))
    a = dict(k_pages=k, v_pages=v, ikey_pages=None, block_table=torch.zeros((1, 4), dtype=torch.int32),
             seq_lens=torch.zeros(1, dtype=torch.int32), kv_scales=torch.zeros((6, 2, 64, 16), dtype=torch.uint8))
    a.update(over)
    return rb.make_cache(**a)


def _wide(n=6):
    return torch.zeros((n, 2, 64, 128), dtype=torch.bfloat16)


def test_the_format_is_what_pages_and_scales_say():
    assert _cache().kv_format == rb.RTP_KV_FP4
    assert _cache(k_pages=_wide(), v_pages=_wide(), kv_scales=None).kv_format == rb.RTP_KV_BF16
    assert _cache(k_pages=_wide().view(torch.int16), v_pages=_wide().view(torch.int16), kv_scales=None).kv_format == rb.RTP_KV_BF16
    ik = torch.zeros((6, 1, 64, 16), dtype=torch.bfloat16)
    assert _cache(k_pages=None, v_pages=None, ikey_pages=ik, kv_scales=None).num_pages == 6


@pytest.mark.parametrize("over", [
    dict(kv_scales=None), dict(kv_scales=None, k_pages=_wide()), dict(k_pages=_wide(), v_pages=_wide()), dict(v_pages=_wide()),
    dict(kv_scales=torch.zeros((6, 2, 64, 16), dtype=torch.bfloat16)), dict(kv_scales=torch.zeros((5, 2, 64, 16), dtype=torch.uint8)),
    dict(k_local_pages=_wide(), v_local_pages=_wide(), local_block_table=torch.zeros((1, 4), dtype=torch.int32)),
    dict(k_local_pages=torch.zeros((6, 1, 64, 64), dtype=torch.uint8), v_local_pages=torch.zeros((6, 1, 64, 64), dtype=torch.uint8),
         local_block_table=torch.zeros((1, 4), dtype=torch.int32), kv_local_scales=torch.zeros((3, 1, 64, 16), dtype=torch.uint8)),
])
def test_pages_and_scales_that_do_not_belong_together_are_refused(over):
    with pytest.raises(rb.RtpError) as e:
        _cache(**over)
    assert e.value.code == rb.RTP_ERR_INVALID


def test_arrays_that_go_together_have_one_length():
    """Calls that take the length of one array for another's: refused before the library is reached (there is no context here)."""
    one, two, many = (torch.zeros(n, dtype=torch.int32) for n in (1, 2, 6))
    c, ws = _cache(), torch.zeros(1 << 12, dtype=torch.uint8)
    for call, args in ((rb.rtp_kv_expand, (two, None, _wide(6), _wide(5), one)), (rb.rtp_kv_expand, (two, None, _wide(5), _wide(6), one)),
                       (rb.rtp_kv_expand, (two, one, _wide(), _wide(), one)), (rb.rtp_cache_copy_pages, (two, one, one)),
                       (rb.rtp_cache_fork, (many, two, one, one)), (rb.rtp_cache_fork, (two, one, one, one)),
                       (rb.rtp_cache_reserve, (many, two, one, ws, one)), (rb.rtp_cache_reserve, (two, one, one, ws, one)),
                       (rb.rtp_cache_free, (two, one, one)), (rb.rtp_cache_compact, (two, one, ws, one))):
        with pytest.raises(rb.RtpError) as e:
            call(None, None, c, *args)
        assert e.value.code == rb.RTP_ERR_INVALID
    with pytest.raises(rb.RtpError):
        _cache(page_refs=two)
    assert _cache(page_refs=many).page_refs == many.data_ptr()


def test_a_replaced_parameter_block_is_the_one_that_calls_take():
    from paper_2605_16928_b200 import build as rbuild
    rbuild.build_library()
    p = rb.Params(8, 2, [], [], [], [])
    before = rb.rtp_workspace_bytes(p, 1, 4096)
    other = rb.Params(8, 2, list(range(8)), [0] * 8, [0], [])
    p.c = other.c
    assert rb.rtp_workspace_bytes(p, 1, 4096) > before
