"""A small 4-bit cache on the device with its decoded values on the host, and the error bounds of the attention over it."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv4_oracle as k4
from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import synth

DEV = "cuda:0"


def dev_bf16(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(synth.to_bf16(np.asarray(x, np.float32)).view(np.int16)).to(DEV).view(torch.bfloat16)


def dev_i32(x) -> torch.Tensor:
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Cache4:
    """B sequences of the given lengths in a 4-bit cache, written by the oracle's encoder.  Whatever is not a token of a
    sequence (other pages, the tails of last pages) holds codes and scales that decode to infinities and NaN."""

    def __init__(self, lens, n_kv=2, group=2, seed=0, ret_kv=(0,), local_kv=(), k=None, v=None, table_cols=0, **params):
        rng = np.random.default_rng(seed)
        self.lens, self.n_kv, self.group = list(lens), n_kv, group
        self.n_q = n_kv * group
        B = len(self.lens)
        pages = [-(-n // 64) for n in self.lens]
        W = max(1, max(pages), table_cols)
        N = sum(pages) + 3
        perm = rng.permutation(N)
        self.kc = np.full((N, n_kv, 64, 64), 0xff, np.uint8)
        self.vc = np.full((N, n_kv, 64, 64), 0xff, np.uint8)
        self.sc = np.full((N, n_kv, 64, 16), 0xff, np.uint8)
        self.bt = np.full((B, W), -1, np.int32)
        self.k, self.v = [], []          # decoded, fp64 [L, n_kv, 128]
        at = 0
        for b, n in enumerate(self.lens):
            self.bt[b, :pages[b]] = perm[at:at + pages[b]]
            at += pages[b]
            kb = rng.standard_normal((n, n_kv, 128)) * np.where(np.arange(128) % 29 == 0, 4.0, 1.0) if k is None else k[b]
            vb = rng.standard_normal((n, n_kv, 128)) if v is None else v[b]
            ck, sk = k4.encode(synth.from_bf16(synth.to_bf16(kb.astype(np.float32))).astype(np.float64))
            cv, sv = k4.encode(synth.from_bf16(synth.to_bf16(vb.astype(np.float32))).astype(np.float64))
            self.k.append(k4.decode(ck, sk))
            self.v.append(k4.decode(cv, sv))
            for t in range(n):
                p, o = self.bt[b, t // 64], t % 64
                self.kc[p, :, o], self.vc[p, :, o] = k4.pack(ck[t]), k4.pack(cv[t])
                self.sc[p, :, o, :8], self.sc[p, :, o, 8:] = sk[t], sv[t]
        self.d_k, self.d_v, self.d_s = (torch.from_numpy(x).to(DEV) for x in (self.kc, self.vc, self.sc))
        self.d_bt, self.d_lens = dev_i32(self.bt), dev_i32(self.lens)
        ret = [kv * group + j for kv in ret_kv for j in range(group)]
        self.ret = ret
        self.local_kv = list(local_kv)
        self.params = rb.Params(self.n_q, n_kv, ret, [list(ret_kv).index(h // group) for h in ret], list(ret_kv), self.local_kv, **params)
        self.sm = float(np.float32(self.params.c.sm_scale))
        self.ctx = rb.Context()
        self.cache = rb.make_cache(self.d_k, self.d_v, None, self.d_bt, self.d_lens, kv_scales=self.d_s)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        q = rng.standard_normal((B, self.n_q, 128)).astype(np.float32)
        self.set_rows(q, np.arange(B), np.array(self.lens) - 1)

    def set_rows(self, q, row_seq, row_pos):
        self.q = synth.from_bf16(synth.to_bf16(np.asarray(q, np.float32))).astype(np.float64)
        self.d_q = dev_bf16(q)
        self.row_seq, self.row_pos = np.asarray(row_seq, np.int32), np.asarray(row_pos, np.int32)
        self.d_seq, self.d_pos = dev_i32(self.row_seq), dev_i32(self.row_pos)
        self.R = len(self.row_seq)
        n = max(1 << 16, rb.rtp_workspace_bytes(self.params, self.R, max(1, max(self.lens))))
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        self.out = torch.full((self.R, self.n_q, 128), -77.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((self.R, self.n_q), -77.0, dtype=torch.float32, device=DEV)

    def args(self):
        return self.ctx, self.params, self.cache, self.d_q, self.d_seq, self.d_pos

    def code(self):
        return rb.rtp_check_status(self.ctx, self.status)

    def check(self, heads, set_of, rows=None, out=None, lse=None):
        """set_of(r, h): the tokens of row r and query head h.  Heads that are not listed have to be left as they were."""
        out = (self.out if out is None else out).double().cpu().numpy()
        lse = (self.lse if lse is None else lse).double().cpu().numpy()
        for r in range(self.R) if rows is None else rows:
            for h in range(self.n_q):
                if h not in heads:
                    assert (out[r, h] == -77.0).all() and lse[r, h] == -77.0, (r, h)
                    continue
                t = np.asarray(set_of(r, h), np.int64)
                b, kv = int(self.row_seq[r]), h // self.group
                if len(t) == 0:
                    assert (out[r, h] == 0).all() and lse[r, h] == -np.inf, (r, h)
                    continue
                o, l, pv, big = k4.attention(self.q[r, h], self.k[b][t, kv], self.v[b][t, kv], self.sm)
                # log2 units: eight fp32 accumulation steps of 2^-23 of sum |q k| each, two products and a difference of 2^-24
                # of it, exp2 2^-22; numerator and denominator both carry it.  Probabilities are rounded to fp16 (2^-11, or
                # 2^-32 absolute where they are subnormal); sums of up to 2^9 terms in fp32: 2^-15.
                a = big * 1.4427
                p_err = 2.0 ** -11 + 2.0 ** -14 + 2.0 ** -17 * a
                tol = 2.0 ** -8 * np.abs(o) + p_err * pv + len(t) * 2.0 ** -32 * np.abs(self.v[b][t, kv]).max()
                assert (np.abs(out[r, h] - o) <= tol).all(), (r, h, len(t), np.abs(out[r, h] - o).max(), tol.min())
                assert abs(lse[r, h] - l) <= 2.0 ** -17 * a + 2.0 ** -14 + 2.0 ** -22 * abs(l), (r, h, lse[r, h], l)
