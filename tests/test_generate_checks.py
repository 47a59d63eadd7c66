"""What the binding of the calls around generation refuses before the library is reached (arrays on the CPU, no context)."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild
from paper_2605_16928_b200 import pipeline


@pytest.fixture()
def params():
    rbuild.build_library()
    return rb.Params(4, 2, [], [], [], [1])


def _i32(*n):
    return torch.zeros(n, dtype=torch.int32)


def _rows(n, heads, dtype=torch.bfloat16):
    return torch.zeros((n, heads, 128), dtype=dtype)


def refused(call):
    with pytest.raises(rb.RtpError) as e:
        call()
    assert e.value.code == rb.RTP_ERR_INVALID


@pytest.mark.parametrize("over", [
    dict(q=None), dict(q_out=None), dict(q=_rows(5, 4)), dict(q=_rows(6, 3)), dict(k=_rows(6, 4)), dict(k=_rows(6, 2, torch.float32)),
    dict(v=_rows(6, 2)[:, :, ::2]), dict(v=_rows(6, 2, torch.float32)[:, :, :64]), dict(k=_rows(2, 6).transpose(0, 1)), dict(tok_pos=_i32(5)),
    dict(q_out=_rows(6, 8)[:, :4]), dict(v=_rows(6, 2)[0]),
])
def test_rotated_appends(params, over):
    a = dict(q=_rows(6, 4), k=_rows(6, 2), v=_rows(6, 2), q_out=_rows(6, 4), w_k=None, tok_seq=_i32(6), tok_pos=_i32(6))
    a.update(over)
    refused(lambda: rb.rtp_rope_append(None, params, None, rb.Rope(torch.zeros(64, dtype=torch.float64)), status=_i32(1), **a))


@pytest.mark.parametrize("over", [
    dict(chunk_start=_i32(2)), dict(row_offsets=_i32(3)), dict(out=_rows(8, 4)), dict(lse=torch.zeros((8, 4))), dict(q=_rows(9, 3)),
    dict(q=_rows(9, 4, torch.float32)), dict(out=_rows(9, 8)[:, :4]), dict(q=_rows(9, 4)[:, :, :64]), dict(lse=torch.zeros((4, 9)).T),
    dict(lse=torch.zeros((9, 4), dtype=torch.float64)), dict(chunk_seq=torch.zeros(3, dtype=torch.int64)), dict(row_offsets=torch.zeros(4, dtype=torch.int64)),
])
def test_chunks(params, over):
    a = dict(q=_rows(9, 4), chunk_seq=_i32(3), chunk_start=_i32(3), row_offsets=_i32(4), pattern=rb.RTP_CHUNK_DENSE, kv_heads=None, out=_rows(9, 4),
             lse=torch.zeros((9, 4)), workspace=torch.zeros(1 << 12, dtype=torch.uint8), status=_i32(1))
    a.update(over)
    refused(lambda: rb.rtp_attn_chunks(None, params, None, **a))


@pytest.mark.parametrize("over", [
    dict(logits=torch.zeros((7, 50))), dict(logits=torch.zeros((6, 50), dtype=torch.float64)), dict(logits=torch.zeros((50, 6)).T),
    dict(scores=torch.zeros(5)), dict(scores=torch.zeros(6, dtype=torch.bfloat16)), dict(finished=_i32(7)), dict(finished=torch.zeros(6, dtype=torch.bool)),
    dict(parent=_i32(4, 2).T), dict(token=_i32(2, 5)), dict(scores_out=torch.zeros((2, 4), dtype=torch.float64)), dict(scores=torch.zeros(12)[::2]),
])
def test_selection(over):
    a = dict(logits=torch.zeros((6, 50)), scores=torch.zeros(6), finished=_i32(6), pad_token=0, parent=_i32(2, 4), token=_i32(2, 4),
             scores_out=torch.zeros((2, 4)), workspace=torch.zeros(1 << 12, dtype=torch.uint8), status=_i32(1))
    a.update(over)
    refused(lambda: rb.rtp_beam_select(None, **a))


def test_reordering(params):
    cache = rb.make_cache(*(torch.zeros((6, 2, 64, 128), dtype=torch.bfloat16) for _ in range(2)), None, _i32(3, 4), _i32(3))
    refused(lambda: rb.rtp_cache_reorder(None, params, cache, _i32(6), _i32(2), _i32(3), _i32(1)))
    refused(lambda: rb.rtp_cache_reorder(None, params, cache, _i32(5), _i32(2), _i32(2), _i32(1)))


@pytest.mark.parametrize("over", [dict(heads=3), dict(rotary_dim=100), dict(rotary_dim=0), dict(rotary_dim=130), dict(dtype=torch.float32)])
def test_frequencies(over):
    n = over.get("heads", 64)
    refused(lambda: rb.Rope(torch.zeros(n, dtype=over.get("dtype", torch.float64)), over.get("rotary_dim", 128)))


def test_beam_path(params, monkeypatch):
    monkeypatch.setattr(rb, "Context", lambda: None)

    def pool(batch=6, arrays=True):
        p = pipeline.PagePool(params, num_pages=10, batch=batch, max_pages=4, device="cpu")
        if arrays:
            p.cache_of(*(torch.zeros((10, 2, 64, 128), dtype=torch.bfloat16) for _ in range(2)))
        return p

    rope = rb.Rope(torch.zeros(64, dtype=torch.float64))
    path = pipeline.BeamPath([pool()], rope, 2, 3, 100, 20)
    assert path.tokens.shape == (2, 3)
    for args in (([pool(5)], rope, 2, 3, 100, 20), ([pool(6, False)], rope, 2, 3, 100, 20), ([pool()], rope, 2, 3, 2, 20), ([pool()], rope, 2, 0, 100, 20),
                 ([pool(70)], rope, 1, 65, 100, 20), ([pool()], rope, 0, 3, 100, 20)):
        refused(lambda: pipeline.BeamPath(*args))
    for lengths in ([4], [4, 0], [15, 6], [1, 2, 3]):
        refused(lambda: path.prompts(lengths))
    refused(lambda: path.begin(torch.zeros((3, 100))))
    refused(lambda: path.begin(torch.zeros((2, 99))))
    refused(lambda: path.choose(torch.zeros((2, 100))))
