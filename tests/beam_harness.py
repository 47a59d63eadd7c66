"""A small model around BeamPath, and the check of its calls against 64 bits."""
import numpy as np
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import pipeline

DEV, VOCAB, LAYERS, N_KV, GROUP = "cuda:0", 700, 2, 2, 2
N_Q, WINDOW, SINKS, LOCAL, END = N_KV * GROUP, 40, 4, 1, 5


class Toy:
    """A model of two layers whose rows depend on the token alone, and whose logits are a fixed projection of the attention."""

    def __init__(self, beams, prompts, pages=None):
        g = torch.Generator(device=DEV)
        g.manual_seed(11)
        self.rows = [torch.randn((VOCAB, N_Q + 2 * N_KV, 128), device=DEV, generator=g).bfloat16() for _ in range(LAYERS)]
        self.head = torch.randn((LAYERS * N_Q * 128, VOCAB), device=DEV, generator=g) * 0.2
        self.prompt = [torch.randint(6, VOCAB, (n,), device=DEV, generator=g) for n in prompts]
        self.freqs = 10000.0 ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64)
        B, cols = len(prompts) * beams, max(prompts) // 64 + 2
        n = pages or B * cols
        self.pools, self.kv = [], []
        for _ in range(LAYERS):
            pool = pipeline.PagePool(rb.Params(N_Q, N_KV, [], [], [], [LOCAL], n_sink=SINKS, window=WINDOW), n, B, cols)
            self.kv.append([torch.full((n, N_KV, 64, 128), torch.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)])
            pool.cache_of(*self.kv[-1])
            self.pools.append(pool)
        self.path = pipeline.BeamPath(self.pools, rb.Rope(self.freqs), len(prompts), beams, VOCAB, sum(prompts), pad_token=0, end_token=END)

    def attend(self, tokens):
        self.outs, self.lses = [], []
        for layer in range(LAYERS):
            x = self.rows[layer][tokens]
            lse = torch.empty((len(x), N_Q), device=DEV)
            self.outs.append(self.path.attend(layer, x[:, :N_Q], x[:, N_Q:N_Q + N_KV], x[:, N_Q + N_KV:], lse=lse))
            self.lses.append(lse)
        return self.outs

    def logits(self, rows=None):
        return torch.cat([(o if rows is None else o[rows]).flatten(1) for o in self.outs], 1).float() @ self.head

    def start(self):
        self.path.prompts([len(p) for p in self.prompt])
        self.attend(torch.cat(self.prompt))
        last = torch.cumsum(torch.tensor([len(p) for p in self.prompt], device=DEV), 0) - 1
        self.first = self.logits(last)
        self.path.begin(self.first)

    def step(self):
        self.path.advance()
        self.attend(self.path.tokens.view(-1).long())
        self.last = self.logits()
        self.path.choose(self.last)

    def check_layer(self, layer, seqs, tokens, pos0):
        """Row i of the last call: the sequence seqs[i], whose tokens are tokens[i], from its position pos0[i] on."""
        table, at = self.pools[layer].block_table.cpu().numpy(), 0
        out, lse = self.outs[layer].float().cpu().numpy(), self.lses[layer].cpu().numpy()
        x = self.rows[layer]
        for s, toks, p0 in zip(seqs, tokens, pos0):
            n, ids = len(toks), torch.tensor(toks, device=DEV)
            pages = torch.tensor(table[s, :-(-n // 64)].astype(np.int64), device=DEV)
            k, v = (a[pages].transpose(1, 2).reshape(-1, N_KV, 128)[:n] for a in self.kv[layer])
            # every cached row is its token's, rotated by its position: one rounding to bf16 on top of 32-bit arithmetic (below 2^-21 of |a| + |b|)
            exact, mag = og.rotate(x[ids, N_Q:N_Q + N_KV].float().cpu().numpy(), np.arange(n), self.freqs.cpu().numpy())
            assert (np.abs(k.float().cpu().numpy() - exact) <= 2.0 ** -8 * np.abs(exact) + mag * 2.0 ** -21 + 1e-38).all()
            assert torch.equal(v, x[ids, N_Q + N_KV:])
            pos = np.arange(p0, n)
            q, qm = og.rotate(x[ids[p0:], :N_Q].float().cpu().numpy(), pos, self.freqs.cpu().numpy())
            kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
            for h in range(N_Q):
                o, l, m = og.attend(q[:, h], kf[:, h // GROUP], vf[:, h // GROUP], pos, 128 ** -0.5, WINDOW if h // GROUP == LOCAL else 0, SINKS)
                # the query is rounded to bf16 first (2^-8 of each element, so 2^-8 |q| |k| / sqrt(128) of a logit at most), then as for the
                # attention alone: 130 x 2^-24 of it for the sums, P and the output 2^-8 each, exponents of two 2^-20
                norm = np.linalg.norm(q[:, h], axis=-1) * np.linalg.norm(kf[:, h // GROUP], axis=-1).max() * 128 ** -0.5
                dz = norm * (2.0 ** -8 + 2.0 ** -21 * 2 + 130 * 2.0 ** -24) + 2.0 ** -20
                got, gl = out[at:at + len(pos), h], lse[at:at + len(pos), h]
                tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.2 * dz[:, None]) * m + 1e-30
                assert (np.abs(got - o) <= tol).all() and (np.abs(gl - l) <= dz + 2.0 ** -22 * np.abs(l)).all(), (layer, s, h)
            at += len(pos)
