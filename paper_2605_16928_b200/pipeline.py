"""Call sequences of the hot path over a ``DeviceData`` workload: buffer allocation and the order of
the C-ABI calls only (no arithmetic happens here).

``PrefillPath.run_chunk`` is one chunk of a chunked prefill (append index keys -> top-p thresholds ->
sparse attention on retrieval heads -> sink+window attention on local heads); ``DecodePath.step`` is
one decode step (append index key -> top-p lists -> sparse attention -> local attention), and both
offer the dense comparator.  With ``kv_fp4`` the K/V cache is held in 4 bits: decode reads it as it is, a
prefill chunk runs on its pages expanded to bf16.

``PagePool`` is the device-side bookkeeping of a pool that sequences come to and leave: table, lengths and
reference counts, and the calls that change them.

``BeamPath`` is beam search over such pools: rotated appends, attention over ragged chunks, selection of the
continuations, and the sequences' places after it.
"""
from __future__ import annotations

import itertools

import torch

from . import binding as rb


class _Base:
    def __init__(self, data, max_rows: int, max_len: int, ikey_e4m3: bool = False, kv_fp4: bool = False, **param_over):
        """ikey_e4m3: the index-key cache holds 8-bit floats (16 bytes per token and index head) instead of bf16.
        kv_fp4: the K/V cache is held in 4 bits (144 bytes per token and KV head instead of 512); the workload's K/V rows
        are quantised into it here."""
        self.data = data
        dev = data.q.device
        self.dev = dev
        self.ctx = rb.Context()
        self.params = rb.Params.from_workload(data, **param_over)
        nih = max(1, data.heads.n_index_heads)
        self.ikey_pages = torch.zeros((data.num_pages, nih, 64, 16),
                                      dtype=torch.uint8 if ikey_e4m3 else torch.bfloat16, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        if kv_fp4:
            n_kv = data.heads.n_kv_heads
            self.k4, self.v4 = (torch.zeros((data.num_pages, n_kv, 64, 64), dtype=torch.uint8, device=dev) for _ in range(2))
            self.kv_scales = torch.zeros((data.num_pages, n_kv, 64, 16), dtype=torch.uint8, device=dev)
            self.cache = rb.make_cache(self.k4, self.v4, self.ikey_pages, data.block_table, data.seq_lens, kv_scales=self.kv_scales)
            self._quantise_all()
        else:
            self.cache = rb.make_cache(data.k_pages, data.v_pages, self.ikey_pages, data.block_table, data.seq_lens)
        ws = max(1 << 20, rb.rtp_workspace_bytes(self.params, max_rows, max_len))
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=dev)
        self.n_ret = len(data.heads.ret_q_heads)
        self.Hq = data.heads.n_q_heads

    def _quantise_all(self, step: int = 1 << 15):
        d = self.data
        for seq in range(int(d.seq_lens.shape[0])):
            n = int(d.seq_lens[seq])
            for lo in range(0, n, step):
                hi = min(n, lo + step)
                rows = []
                for pages in (d.k_pages, d.v_pages):
                    x = pages[d.block_table[seq, lo // 64:(hi + 63) // 64].long()].transpose(1, 2)
                    rows.append(x.reshape(-1, d.heads.n_kv_heads, 128)[:hi - lo].contiguous())
                self.append_kv(seq, lo, rows[0], rows[1])

    def append_kv(self, seq: int, lo: int, k_new, v_new):
        """K/V rows of tokens lo .. of a sequence into the cache, in the form it is held in."""
        n = int(k_new.shape[0])
        tok_seq = torch.full((n,), seq, dtype=torch.int32, device=self.dev)
        tok_pos = torch.arange(lo, lo + n, dtype=torch.int32, device=self.dev)
        rb.rtp_kv_append(self.ctx, self.params, self.cache, k_new, v_new, tok_seq, tok_pos, self.status)

    def status_code(self) -> int:
        return rb.rtp_check_status(self.ctx, self.status)

    def index_keys_range(self, seq: int, lo: int, hi: int, k_pre=None):
        d = self.data
        k_pre = d.k_pre_rows(seq, lo, hi) if k_pre is None else k_pre
        tok_seq = torch.full((hi - lo,), seq, dtype=torch.int32, device=self.dev)
        tok_pos = torch.arange(lo, hi, dtype=torch.int32, device=self.dev)
        rb.rtp_index_keys(self.ctx, self.params, self.cache, k_pre, d.w_k, tok_seq, tok_pos)


class PrefillPath(_Base):
    """One sequence, rows = positions.  Buffers are sized for one chunk."""

    def __init__(self, data, chunk: int, kv_fp4: bool = False):
        """kv_fp4: every run_* call expands the pages of the sequence so far to bf16 and attends to those (``attn_cache``);
        the expansion of 128K tokens is about a hundredth of a chunk's dense attention over them.  The bf16 pool stands beside the
        4-bit one for as long as the path does: the saving is the decode's that follows."""
        L = int(data.seq_lens[0])
        super().__init__(data, chunk, L, kv_fp4=kv_fp4)
        self.L, self.chunk = L, chunk
        self.attn_cache = self.cache
        if kv_fp4:   # the same page numbers in a bf16 pool
            self.k_wide, self.v_wide = (torch.zeros((data.num_pages, data.heads.n_kv_heads, 64, 128), dtype=torch.bfloat16,
                                                    device=self.dev) for _ in range(2))
            self.attn_cache = rb.make_cache(self.k_wide, self.v_wide, self.ikey_pages, data.block_table, data.seq_lens)
        self.sel_cnt = torch.empty((chunk, self.n_ret), dtype=torch.int32, device=self.dev)
        self.sel_mass = torch.empty((chunk, self.n_ret), dtype=torch.float32, device=self.dev)
        self.sel_thr = torch.empty((chunk, self.n_ret), dtype=torch.float32, device=self.dev)
        self.sel_tie = torch.empty((chunk, self.n_ret), dtype=torch.int32, device=self.dev)
        self.tok_seq = torch.zeros(chunk, dtype=torch.int32, device=self.dev)
        self.pos_all = torch.arange(L, dtype=torch.int32, device=self.dev)
        self.launches_per_chunk = 6 + kv_fp4   # (expansion,) index_keys, 2 x query projection, select, sparse attention, local attention
        self.blk_mask = None          # block-wise path (Section 3.4): allocated on first use

    def _expand(self, n_tokens: int):
        if self.attn_cache is not self.cache:
            ids = self.data.block_table[0, :(n_tokens + 63) // 64]
            rb.rtp_kv_expand(self.ctx, self.params, self.cache, ids, ids, self.k_wide, self.v_wide, self.status)

    def chunks(self):
        return [(s, min(self.chunk, self.L - s)) for s in range(0, self.L, self.chunk)]

    def run_chunk(self, q_start: int, C: int, q, k_pre, out, lse=None):
        """q: bf16 [C, Hq, 128] (also used as q_pre: no RoPE in the synthetic workloads);
        k_pre: bf16 [C, n_index_heads, 128]; out: bf16 [C, Hq, 128]."""
        d, p = self.data, self.params
        self._expand(q_start + C)
        rb.rtp_index_keys(self.ctx, p, self.cache, k_pre, d.w_k, self.tok_seq[:C], self.pos_all[q_start:q_start + C])
        rb.rtp_topp_select(self.ctx, p, self.cache, q, d.w_q, None, None, 0, q_start, C, None, self.sel_cnt,
                           self.sel_mass, self.sel_thr, self.sel_tie, self.status, self.workspace)
        rb.rtp_sparse_attn_prefill(self.ctx, p, self.attn_cache, q, q, d.w_q, 0, q_start, C, None, self.sel_cnt,
                                   self.sel_thr, self.sel_tie, out, lse, self.workspace, self.status)
        rb.rtp_local_attn(self.ctx, p, self.attn_cache, q, None, None, 0, q_start, C, out, lse, self.workspace, self.status)

    def run_chunk_blocks(self, q_start: int, C: int, q, k_pre, out, lse=None):
        """The same chunk with the block-wise selection of Section 3.4 on the retrieval heads: append index keys ->
        one bit per (row, head, page) -> attention over the selected pages -> sink + window attention on local heads."""
        d, p = self.data, self.params
        self._expand(q_start + C)
        if self.blk_mask is None:
            words = (((self.L + 63) // 64 + 31) // 32 + 3) // 4 * 4
            self.blk_mask = torch.zeros((self.chunk, self.n_ret, words), dtype=torch.int32, device=self.dev)
            self.blk_ws = torch.empty(rb.rtp_block_workspace_bytes(p, self.chunk, self.L), dtype=torch.uint8, device=self.dev)
        rb.rtp_index_keys(self.ctx, p, self.cache, k_pre, d.w_k, self.tok_seq[:C], self.pos_all[q_start:q_start + C])
        rb.rtp_topp_select_blocks(self.ctx, p, self.cache, q, d.w_q, 0, q_start, C, self.blk_mask[:C], self.sel_cnt[:C],
                                  self.sel_mass[:C], self.sel_thr[:C], self.sel_tie[:C], self.status, self.blk_ws)
        rb.rtp_sparse_attn_prefill_blocks(self.ctx, p, self.attn_cache, q, 0, q_start, C, self.blk_mask[:C], out, lse, self.status)
        rb.rtp_local_attn(self.ctx, p, self.attn_cache, q, None, None, 0, q_start, C, out, lse, self.workspace, self.status)

    def run_chunk_dense(self, q_start: int, C: int, q, out, lse=None):
        self._expand(q_start + C)
        rb.rtp_dense_attn_prefill(self.ctx, self.params, self.attn_cache, q, 0, q_start, C, None, out, lse, self.status)


class DecodePath(_Base):
    """One decode step for a batch: row b is the newest token of sequence b."""

    def __init__(self, data, sel_stride: int, **param_over):
        """param_over: rtp_params fields that replace the workload's (top_k, force_sink, force_recent, top_p ...), and the cache
        forms of _Base (ikey_e4m3, kv_fp4)."""
        B = int(data.seq_lens.shape[0])
        L = int(data.seq_lens.max())
        super().__init__(data, B, L, **param_over)
        self.B, self.L = B, L
        self.sel_idx = torch.empty((B, self.n_ret, sel_stride), dtype=torch.int32, device=self.dev)
        self.sel_cnt = torch.empty((B, self.n_ret), dtype=torch.int32, device=self.dev)
        self.sel_mass = torch.empty((B, self.n_ret), dtype=torch.float32, device=self.dev)
        self.sel_thr = torch.empty((B, self.n_ret), dtype=torch.float32, device=self.dev)
        self.sel_tie = torch.empty((B, self.n_ret), dtype=torch.int32, device=self.dev)
        self.out = torch.empty((B, self.Hq, 128), dtype=torch.bfloat16, device=self.dev)
        self.lse = torch.empty((B, self.Hq), dtype=torch.float32, device=self.dev)
        # local heads do not depend on the retrieval heads: their attention runs on a second stream with a workspace
        # of its own and joins before the step returns
        self.side = torch.cuda.Stream(device=self.dev)
        self.workspace_local = torch.empty_like(self.workspace)
        self.has_local = len(data.heads.local_kv_heads) > 0

    def build_index_cache(self, step: int = 1 << 17):
        for b in range(self.B):
            for lo in range(0, self.L, step):
                self.index_keys_range(b, lo, min(self.L, lo + step))

    def step(self, q, k_pre_new):
        """q: bf16 [B, Hq, 128]; k_pre_new: bf16 [B, n_index_heads, 128] pre-RoPE keys of the newest tokens."""
        d, p = self.data, self.params
        main = torch.cuda.current_stream()
        if self.has_local:
            self.side.wait_stream(main)
            rb.rtp_local_attn(self.ctx, p, self.cache, q, d.row_seq, d.row_pos, 0, 0, self.B, self.out, self.lse,
                              self.workspace_local, self.status, stream=self.side)
        rb.rtp_index_keys(self.ctx, p, self.cache, k_pre_new, d.w_k, d.row_seq, d.row_pos)
        rb.rtp_topp_select(self.ctx, p, self.cache, q, d.w_q, d.row_seq, d.row_pos, 0, 0, self.B, self.sel_idx,
                           self.sel_cnt, self.sel_mass, self.sel_thr, self.sel_tie, self.status, self.workspace)
        rb.rtp_sparse_attn_decode(self.ctx, p, self.cache, q, d.row_seq, d.row_pos, self.sel_idx, self.sel_cnt,
                                  self.out, self.lse, self.workspace, self.status)
        if self.has_local:
            main.wait_stream(self.side)

    def step_blocks(self, q, k_pre_new):
        """The same decode step with the block-wise selector of Section 3.4: whole 64-key pages are selected by their
        log-sum-exp mass and attended to.  Buffers are made on first use."""
        d, p = self.data, self.params
        if not hasattr(self, "blk_idx"):
            n_b = (self.L + 63) // 64
            self.blk_idx = torch.empty((self.B, self.n_ret, n_b), dtype=torch.int32, device=self.dev)
            self.blk_cnt = torch.empty((self.B, self.n_ret), dtype=torch.int32, device=self.dev)
            self.blk_ws = torch.empty(max(1 << 16, rb.rtp_block_workspace_bytes(p, self.B, self.L)), dtype=torch.uint8,
                                      device=self.dev)
        main = torch.cuda.current_stream()
        if self.has_local:
            self.side.wait_stream(main)
            rb.rtp_local_attn(self.ctx, p, self.cache, q, d.row_seq, d.row_pos, 0, 0, self.B, self.out, self.lse,
                              self.workspace_local, self.status, stream=self.side)
        rb.rtp_index_keys(self.ctx, p, self.cache, k_pre_new, d.w_k, d.row_seq, d.row_pos)
        rb.rtp_topp_select_blocks_rows(self.ctx, p, self.cache, q, d.w_q, d.row_seq, d.row_pos, self.blk_idx, self.blk_cnt,
                                       self.sel_mass, self.sel_thr, self.sel_tie, self.status, self.blk_ws)
        rb.rtp_sparse_attn_decode_blocks(self.ctx, p, self.cache, q, d.row_seq, d.row_pos, self.blk_idx, self.blk_cnt,
                                         self.out, self.lse, self.workspace, self.status)
        if self.has_local:
            main.wait_stream(self.side)

    def step_dense(self, q):
        d = self.data
        rb.rtp_dense_attn_decode(self.ctx, self.params, self.cache, q, d.row_seq, d.row_pos, None, self.out, self.lse,
                                 self.workspace, self.status)


class PagePool:
    """Block table, sequence lengths and reference counts of a pool of pages, on the device.  ``cache_of`` gives the arrays of
    the pool the description that the other calls take; every method is one call in stream order, nothing is read back.  The
    description names the reference counts, so that appends leave pages alone that sequences share (after a reserve that found
    the pool full, for instance).
    ``status`` collects what only the device can see (a full pool: RTP_ERR_CAPACITY) until ``status_code`` reads it."""

    def __init__(self, params: rb.Params, num_pages: int, batch: int, max_pages: int, device="cuda:0"):
        dev = torch.device(device)
        if dev.type == "cuda" and dev.index is not None and dev.index != torch.cuda.current_device():
            raise rb.RtpError(rb.RTP_ERR_INVALID, "PagePool", f"{dev} is not the current device, on which the calls run")
        i32 = dict(dtype=torch.int32, device=device)
        self.ctx, self.params = rb.Context(), params
        self.block_table = torch.full((batch, max_pages), -1, **i32)
        self.seq_lens = torch.zeros(batch, **i32)
        self.page_refs = torch.zeros(num_pages, **i32)
        self.n_used = torch.zeros(1, **i32)
        self.status = torch.zeros(1, **i32)
        self.cache = self.workspace = None

    def cache_of(self, k_pages, v_pages, ikey_pages=None, kv_scales=None) -> rb.RtpCache:
        """Arrays [num_pages, heads, 64, ..] on the pool's device: K and V with the parameter block's KV heads, index keys with
        its index heads; None for what the cache does not hold.  A pool is one set of arrays: reserve and compact copy the pages of
        those named last, so every layer has a pool of its own."""
        for name, x, heads in (("k_pages", k_pages, self.params.c.n_kv_heads), ("v_pages", v_pages, self.params.c.n_kv_heads),
                               ("ikey_pages", ikey_pages, self.params.c.n_index_heads),
                               ("kv_scales", kv_scales, self.params.c.n_kv_heads)):
            if x is None:
                continue
            want = (self.page_refs.numel(), heads)
            if tuple(x.shape[:2]) != want or x.device != self.page_refs.device or not x.is_contiguous():
                raise rb.RtpError(rb.RTP_ERR_INVALID, "PagePool.cache_of",
                                  f"{name} has to be a contiguous array of {want[0]} pages of {want[1]} heads on {self.page_refs.device}")
        self.cache = rb.make_cache(k_pages, v_pages, ikey_pages, self.block_table, self.seq_lens, kv_scales=kv_scales,
                                   page_refs=self.page_refs)
        self.workspace = torch.empty(rb.rtp_cache_workspace_bytes(self.cache, min(4096, int(self.seq_lens.shape[0]))),
                                     dtype=torch.uint8, device=self.seq_lens.device)
        return self.cache

    def reserve(self, seqs, n_tokens):
        rb.rtp_cache_reserve(self.ctx, self.params, self.cache, self.page_refs, seqs, n_tokens, self.workspace, self.status)

    def fork(self, src_seqs, dst_seqs):
        rb.rtp_cache_fork(self.ctx, self.params, self.cache, self.page_refs, src_seqs, dst_seqs, self.status)

    def reorder(self, src_seqs, dst_seqs):
        """Sequence dst_seqs[i] becomes what src_seqs[i] was, all at once."""
        rb.rtp_cache_reorder(self.ctx, self.params, self.cache, self.page_refs, src_seqs, dst_seqs, self.status)

    def free(self, seqs):
        rb.rtp_cache_free(self.ctx, self.params, self.cache, self.page_refs, seqs, self.status)

    def compact(self):
        rb.rtp_cache_compact(self.ctx, self.params, self.cache, self.page_refs, self.n_used, self.workspace, self.status)

    def status_code(self) -> int:
        """The largest code recorded since the last call of this method, which clears it."""
        code = rb.rtp_check_status(self.ctx, self.status)
        if code != rb.RTP_OK:
            self.status.zero_()
        return code


class BeamPath:
    """Beam search over page pools, one per layer: sequence g * n_beams + b of every pool is hypothesis b of group g.

        path.prompts(lengths); out = path.attend(layer, q, k, v) for every layer; path.begin(logits of each prompt's last row)
        path.advance();        out = path.attend(layer, q, k, v) for every layer; path.choose(logits of the hypotheses)      (a step)

    ``tokens`` [groups x beams] are the tokens to go on with, ``parents`` the rows that they continue (of a first choice: row
    g * n_beams, where the prompt lies), ``scores`` the sums of log-probabilities and ``finished`` what has ended with ``end_token``.
    Nothing is read back; a step writes to the same arrays every time and may be captured into a graph.  Its shape is the same every
    time, too: a hypothesis that has ended goes on taking room, with ``pad_token``.

    ``status`` as in PagePool.  Where a pool has something to report after its pages were asked for (it is full: RTP_ERR_CAPACITY),
    no sequence of any pool grows, by ``prompts`` or ``advance``, until ``status_code`` has read and cleared it: the call can be made
    again when sequences have been freed.  What follows a call that failed is not to be used."""

    def __init__(self, pools, rope: rb.Rope, n_groups: int, n_beams: int, vocab: int, max_rows: int, pattern: int = rb.RTP_CHUNK_BY_HEAD,
                 pad_token: int = 0, end_token: int = -1):
        """max_rows: of all prompts together."""
        B, first = n_groups * n_beams, pools[0]
        if any(p.seq_lens.shape[0] < B or p.cache is None for p in pools) or not 1 <= n_beams <= min(vocab, rb.RTP_MAX_BEAMS) or n_groups < 1:
            raise rb.RtpError(rb.RTP_ERR_INVALID, "BeamPath", f"pools of {B} sequences with their arrays, 1 <= beams <= {rb.RTP_MAX_BEAMS} and the vocabulary")
        if any(p.cache.kv_format != rb.RTP_KV_BF16 for p in pools):
            raise rb.RtpError(rb.RTP_ERR_UNSUPPORTED, "BeamPath", "a 4-bit pool: its attention (rtp_attn_chunks) reads bf16 pages")
        self.pools, self.rope, self.pattern, self.pad_token, self.end_token = list(pools), rope, pattern, pad_token, end_token
        self.ctx, self.n_groups, self.n_beams, self.vocab, self.max_rows = rb.Context(), n_groups, n_beams, vocab, max(max_rows, B)
        dev = first.seq_lens.device
        i32 = dict(dtype=torch.int32, device=dev)
        self.dev, self.status = dev, torch.zeros(1, **i32)
        self.seqs, self.ones = torch.arange(B, **i32), torch.ones(B, **i32)
        self.positions, self.offsets = torch.zeros(B, **i32), torch.arange(B + 1, **i32)
        self.tokens, self.parents, self.finished = (torch.zeros((n_groups, n_beams), **i32) for _ in range(3))
        self.scores, self._scores = (torch.zeros((n_groups, n_beams), dtype=torch.float32, device=dev) for _ in range(2))
        heads = max(p.params.c.n_q_heads for p in pools)
        self.q = torch.empty((self.max_rows, heads, 128), dtype=torch.bfloat16, device=dev)
        ws = max([rb.rtp_chunk_workspace_bytes(p.params, B, self.max_rows) for p in pools] + [rb.rtp_beam_workspace_bytes(B, vocab, n_beams)])
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=dev)
        self.batch = None

    def _granted(self):
        """[1], on the device: 1 if no pool has anything to report, else 0."""
        status = self.pools[0].status if len(self.pools) == 1 else torch.cat([p.status for p in self.pools]).amax(0, keepdim=True)
        return (status == rb.RTP_OK).int()

    def prompts(self, lengths):
        """One prompt a group, by its number of tokens: pages for them in every pool.  The sequences have to be empty."""
        if len(lengths) != self.n_groups or min(lengths) < 1 or sum(lengths) > self.max_rows:
            raise rb.RtpError(rb.RTP_ERR_INVALID, "BeamPath.prompts", f"{self.n_groups} lengths of at least one, at most {self.max_rows} in all")
        i32 = dict(dtype=torch.int32, device=self.dev)
        seqs, n = self.seqs[::self.n_beams].contiguous(), torch.tensor(lengths, **i32)
        for p in self.pools:
            p.reserve(seqs, n)
        granted = n * self._granted()
        for p in self.pools:
            p.seq_lens[:self.seqs.shape[0]:self.n_beams] = granted
        self.batch = (seqs, torch.zeros(self.n_groups, **i32), torch.tensor([0, *itertools.accumulate(lengths)], **i32),
                      torch.repeat_interleave(seqs, n, output_size=sum(lengths)), torch.cat([torch.arange(x, **i32) for x in lengths]))

    def advance(self):
        """Room for one token of every hypothesis, behind its last one."""
        self.positions.copy_(self.pools[0].seq_lens[:self.seqs.shape[0]])
        for p in self.pools:
            p.reserve(self.seqs, self.ones)
        granted = self._granted()
        for p in self.pools:
            p.seq_lens[:self.seqs.shape[0]] += granted
        self.batch = (self.seqs, self.positions, self.offsets, self.seqs, self.positions)

    def attend(self, layer: int, q, k, v, out=None, lse=None, w_k=None):
        """The batch's rows of one layer as the projections leave them: rotated and appended, then attended over their sequences."""
        pool = self.pools[layer]
        seq, start, offsets, tok_seq, tok_pos = self.batch
        q_rot = self.q.view(-1)[:q.shape[0] * q.shape[1] * 128].view(q.shape[0], q.shape[1], 128)
        out = torch.empty_like(q_rot) if out is None else out
        rb.rtp_rope_append(self.ctx, pool.params, pool.cache, self.rope, q, k, v, q_rot, w_k, tok_seq, tok_pos, self.status)
        rb.rtp_attn_chunks(self.ctx, pool.params, pool.cache, q_rot, seq, start, offsets, self.pattern, None, out, lse, self.workspace, self.status)
        return out

    def _select(self, logits, scores, finished):
        if logits.shape[1] != self.vocab:
            raise rb.RtpError(rb.RTP_ERR_INVALID, "BeamPath", f"logits over {logits.shape[1]} tokens, not {self.vocab}")
        rb.rtp_beam_select(self.ctx, logits, scores, finished, self.pad_token, self.parents, self.tokens, self._scores, self.workspace, self.status)
        self.scores.copy_(self._scores)

    def begin(self, logits):
        """logits [groups, vocabulary] behind the prompts: the best tokens begin the hypotheses, which share their prompt's pages."""
        if logits.shape[0] != self.n_groups:
            raise rb.RtpError(rb.RTP_ERR_INVALID, "BeamPath.begin", f"logits of {logits.shape[0]} rows, not of {self.n_groups}")
        self._select(logits, None, None)
        self.parents.mul_(self.n_beams)            # (the selection's rows were the groups)
        if self.n_beams > 1:
            src = self.seqs.view(self.n_groups, self.n_beams)[:, :1].expand(-1, self.n_beams - 1).contiguous().view(-1)
            dst = self.seqs.view(self.n_groups, self.n_beams)[:, 1:].contiguous().view(-1)
            for p in self.pools:
                p.fork(src, dst)
        self.finished.copy_(self.tokens == self.end_token)

    def choose(self, logits):
        """logits [groups x beams, vocabulary]: the best continuations take the hypotheses' places, with their sequences."""
        if logits.shape[0] != self.seqs.shape[0]:
            raise rb.RtpError(rb.RTP_ERR_INVALID, "BeamPath.choose", f"logits of {logits.shape[0]} rows, not of {self.seqs.shape[0]}")
        self._select(logits, self.scores, self.finished)
        parents = self.parents.view(-1)
        for p in self.pools:
            p.reorder(parents, self.seqs)
        ended = self.finished.view(-1)[parents.clamp(min=0)].view_as(self.finished)
        torch.maximum(ended, (self.tokens == self.end_token).int(), out=self.finished)

    def status_code(self) -> int:
        """The largest code that its own calls and its pools' have recorded since the last call of this method."""
        code = rb.rtp_check_status(self.ctx, self.status)
        if code != rb.RTP_OK:
            self.status.zero_()
        return max([code] + [p.status_code() for p in self.pools])
