"""What the binding of the calls around generation refuses by type, shape or device (arrays on the CPU, no context): an array that the
library would take for something else, or read beyond its end."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import build as rbuild
from tests.test_generate_checks import _i32, _rows, refused

F16 = torch.float16


@pytest.fixture()
def params():
    rbuild.build_library()
    return rb.Params(4, 2, [0, 2], [0, 1], [0, 1], [])


@pytest.mark.parametrize("over", [
    dict(w_k=torch.zeros((1, 128, 16), dtype=torch.bfloat16)), dict(w_k=torch.zeros((2, 128, 8), dtype=torch.bfloat16)),
    dict(w_k=torch.zeros((2, 128, 16), dtype=F16)), dict(w_k=torch.zeros((2, 128, 16))), dict(w_k=torch.zeros((2, 16, 128), dtype=torch.bfloat16).transpose(1, 2)),
    dict(w_k=torch.zeros((2, 128, 32), dtype=torch.bfloat16)[:, :, ::2]), dict(w_k=torch.zeros((2, 128, 16), dtype=torch.bfloat16, device="meta")),
    dict(q=_rows(6, 4, F16)), dict(q_out=_rows(6, 4, F16)), dict(k=_rows(6, 2, F16)), dict(v=_rows(6, 2, F16)), dict(v=_rows(6, 2, torch.int16)),
    dict(tok_pos=torch.zeros(6)), dict(tok_seq=torch.zeros(6)),
])
def test_rotated_appends(params, over):
    a = dict(q=_rows(6, 4), k=_rows(6, 2), v=_rows(6, 2), q_out=_rows(6, 4), w_k=torch.zeros((2, 128, 16), dtype=torch.bfloat16), tok_seq=_i32(6), tok_pos=_i32(6))
    a.update(over)
    refused(lambda: rb.rtp_rope_append(None, params, None, rb.Rope(torch.zeros(64, dtype=torch.float64)), status=_i32(1), **a))


def test_frequencies_on_another_device(params):
    a = dict(q=None, k=_rows(6, 2), v=_rows(6, 2), q_out=None, w_k=None, tok_seq=_i32(6), tok_pos=_i32(6), status=_i32(1))
    refused(lambda: rb.rtp_rope_append(None, params, None, rb.Rope(torch.zeros(64, dtype=torch.float64, device="meta")), **a))
    with pytest.raises(AttributeError):            # (all else is right: only the context is missing)
        rb.rtp_rope_append(None, params, None, rb.Rope(torch.zeros(64, dtype=torch.float64)), **a)


@pytest.mark.parametrize("over", [
    dict(q=_rows(9, 4, F16)), dict(out=_rows(9, 4, F16)), dict(q=_rows(9, 4, torch.int16)), dict(lse=_i32(9, 4)), dict(chunk_seq=torch.zeros(3)),
    dict(chunk_start=torch.zeros(3)), dict(row_offsets=torch.zeros(4)),
])
def test_chunks(params, over):
    a = dict(q=_rows(9, 4), chunk_seq=_i32(3), chunk_start=_i32(3), row_offsets=_i32(4), pattern=rb.RTP_CHUNK_DENSE, kv_heads=None, out=_rows(9, 4),
             lse=torch.zeros((9, 4)), workspace=torch.zeros(1 << 12, dtype=torch.uint8), status=_i32(1))
    a.update(over)
    refused(lambda: rb.rtp_attn_chunks(None, params, None, **a))


@pytest.mark.parametrize("over", [
    dict(scores=_i32(6)), dict(finished=torch.zeros(6)), dict(parent=torch.zeros((2, 4))), dict(token=torch.zeros((2, 4))), dict(scores_out=_i32(2, 4)),
    dict(logits=torch.zeros((6, 50), dtype=torch.int32)), dict(logits=torch.zeros((6, 50), dtype=torch.int16)),
])
def test_selection(over):
    a = dict(logits=torch.zeros((6, 50)), scores=torch.zeros(6), finished=_i32(6), pad_token=0, parent=_i32(2, 4), token=_i32(2, 4),
             scores_out=torch.zeros((2, 4)), workspace=torch.zeros(1 << 12, dtype=torch.uint8), status=_i32(1))
    a.update(over)
    refused(lambda: rb.rtp_beam_select(None, **a))


@pytest.mark.parametrize("which", ["page_refs", "src_seqs", "dst_seqs"])
def test_reordering(params, which):
    cache = rb.make_cache(*(torch.zeros((6, 2, 64, 128), dtype=torch.bfloat16) for _ in range(2)), None, _i32(3, 4), _i32(3))
    a = dict(page_refs=_i32(6), src_seqs=_i32(2), dst_seqs=_i32(2), status=_i32(1))
    a[which] = a[which].float()
    refused(lambda: rb.rtp_cache_reorder(None, params, cache, **a))
