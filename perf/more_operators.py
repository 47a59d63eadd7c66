"""Measured cases of the calls that a program makes around the attention when it generates text from several prompts or with
several hypotheses a prompt.

Operators:
  append   queries and keys rotated by their positions, keys and values put into their pages, index keys of the unrotated keys
           (``rtp_rope_append``)
  chunks   attention of pieces of several sequences, of one row up to thousands, over their pages (``rtp_attn_chunks``)
  beam     the k best continuations over the beams and the vocabulary of each group (``rtp_beam_select``)
  reorder  sequences take over the pages of the hypotheses that survive (``rtp_cache_reorder``)
"""
import math

import numpy as np
import torch

own = False

PAGE, DIM, IDX = 64, 128, 16


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a batch of sixteen on a bf16 cache with two index heads
        dict(name="append_step_b16", kind="append", B=16, T=16, L=32768, Hkv=8, group=4, rd=128, inter=False, n_ih=2, e4m3=False),
        # an 8192-token chunk of a long prompt
        dict(name="append_chunk_8k_of_128k", kind="append", B=1, T=8192, L=131072, Hkv=8, group=4, rd=128, inter=False, n_ih=2, e4m3=False),
        # pieces of five prompts, half of the channels rotated in neighbouring pairs, 8-bit index keys
        dict(name="append_ragged_1003", kind="append", B=5, T=1003, L=9001, Hkv=4, group=3, rd=64, inter=True, n_ih=1, e4m3=True),
        # a question of seven tokens behind a short conversation
        dict(name="chunk_7_of_200", kind="chunks", n=1, rows=7, keys=200, Hkv=8, group=4, by_head=False, n_loc=0, window=2048),
        # five proposed tokens verified for each of 32 conversations
        dict(name="chunks_verify_32x5", kind="chunks", n=32, rows=5, keys=8192, Hkv=8, group=4, by_head=False, n_loc=0, window=2048),
        # a serving step: decode rows and pieces of prompts together, six of eight KV heads with sinks and a window
        dict(name="chunks_mixed_12", kind="chunks", n=12, rows=700, keys=32768, Hkv=8, group=4, by_head=True, n_loc=6, window=2048),
        # a chunk of 2048 prompt tokens over 32K, every head over everything
        dict(name="chunk_2k_of_32k", kind="chunks", n=1, rows=2048, keys=32768, Hkv=8, group=4, by_head=False, n_loc=0, window=2048),
        # one request with four beams
        dict(name="beam_1x4_32k", kind="beam", G=1, W=4, V=32768, K=8, f32=False, done=0.0, masked=0.0),
        # requests with odd sizes in 32 bits: some beams have ended, most of the vocabulary is ruled out
        dict(name="beam_5x3_50001", kind="beam", G=5, W=3, V=50001, K=6, f32=True, done=0.2, masked=0.9),
        # a batch of 32 requests with eight beams each over a large vocabulary
        dict(name="beam_32x8_128k", kind="beam", G=32, W=8, V=131072, K=16, f32=False, done=0.05, masked=0.0),
        # four beams of one conversation
        dict(name="reorder_1x4_4k", kind="reorder", G=1, W=4, L=4099, tail=100),
        # eight beams each of 32 requests with long prompts
        dict(name="reorder_32x8_32k", kind="reorder", G=32, W=8, L=32803, tail=900),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["append", "chunks", "chunks", "beam", "beam", "reorder"])
    if kind == "append":
        Hkv = rng.choice([1, 2, 4, 8])
        L, T = _log(rng, 64, 131072), _log(rng, 1, 8192)
        B = rng.randint(1, min(16, T))
        return dict(kind=kind, B=B, T=min(T, B * L), L=L, Hkv=Hkv, group=rng.randint(1, 32 // Hkv) if Hkv > 4 else rng.randint(1, 8),
                    rd=rng.choice([32, 64, 96, 128, 128, 128]), inter=rng.random() < 0.3, n_ih=rng.randint(0, min(2, Hkv)), e4m3=rng.random() < 0.3)
    if kind == "chunks":
        Hkv = rng.choice([1, 2, 4, 8])
        by_head = Hkv > 1 and rng.random() < 0.4
        keys = _log(rng, 1, 32768)
        rows = _log(rng, 1, 2048)
        # (no more query rows times keys, padded to the longest of the batch, and no more keys than the largest listed cases)
        n = rng.randint(1, max(1, min(32, 2048 * 32768 // (min(rows, keys) * keys), 1000000 // (keys * Hkv))))
        return dict(kind=kind, n=n, rows=min(rows, keys), keys=keys, Hkv=Hkv, group=rng.randint(1, 32 // Hkv) if Hkv > 4 else rng.choice([1, 2, 3, 4, 6, 8]),
                    by_head=by_head, n_loc=rng.randint(1, Hkv - 1) if by_head else 0, window=_log(rng, 16, 4096))
    if kind == "beam":
        V, W = _log(rng, 100, 131072), rng.randint(1, 16)
        G = rng.randint(1, max(1, min(64, 32 * 8 * 131072 // (2 * V * W))))
        return dict(kind=kind, G=G, W=W, V=V, K=rng.randint(1, 32), f32=rng.random() < 0.5, done=rng.choice([0.0, 0.2]), masked=rng.choice([0.0, 0.0, 0.9]))
    return dict(kind=kind, G=_log(rng, 1, 32), W=rng.randint(1, 8), L=_log(rng, 1, 32768), tail=_log(rng, 1, 1000))


def _parts(total, n):
    """`total` cut into n uneven pieces of at least one."""
    w = [1.0 + (5 * i % 7) for i in range(n)]
    cut = [int(total * sum(w[:i]) / sum(w)) for i in range(n + 1)]
    p = [max(1, cut[i + 1] - cut[i]) for i in range(n)]
    p[0] += total - sum(p)
    return p if p[0] > 0 else [total // n + (i < total % n) for i in range(n)]


def _chunks(c):
    """(rows, keys) of each chunk: the first the longest; the others shrink to an eighth and, every third one, to single rows where
    the chunks are long ones."""
    out = []
    for i in range(c["n"]):
        keys = max(1, c["keys"] - (i * 2657) % (c["keys"] * 7 // 8 + 1))
        rows = c["rows"] if c["rows"] <= 8 or i == 0 else 1 if i % 3 == 1 else max(1, c["rows"] >> (i % 6))
        out.append((min(rows, keys), keys))
    return out


def _seen(c, m, local):
    """Keys that a row at position m attends to."""
    if not local or m + 1 <= c["window"]:
        return m + 1
    return c["window"] + min(4, m + 1 - c["window"])


def work(c):
    if c["kind"] == "append":
        Hq = c["Hkv"] * c["group"]
        row = 2 * (Hq + 2 * c["Hkv"]) * DIM
        return {"bytes": c["T"] * (2 * row + c["n_ih"] * IDX * (1 if c["e4m3"] else 2) + 8), "flops": c["T"] * ((Hq + c["Hkv"]) * 3 * c["rd"] + c["n_ih"] * 2 * DIM * IDX)}
    if c["kind"] == "chunks":
        toks = pairs = rows = 0
        for r, n in _chunks(c):
            rows += r
            for local, heads in ((False, c["Hkv"] - c["n_loc"]), (True, c["n_loc"])):
                pairs += heads * sum(_seen(c, m, local) for m in range(n - r, n))
                first = max(0, n - r - c["window"] + 1) if local else 0
                toks += heads * (n - first + min(4, first))
        Hq = c["Hkv"] * c["group"]
        return {"bytes": toks * 4 * DIM + rows * Hq * (4 * DIM + 4), "flops": pairs * c["group"] * 4 * DIM}
    if c["kind"] == "beam":
        n = c["G"] * c["W"]
        return {"bytes": n * c["V"] * (4 if c["f32"] else 2) + n * 8 + c["G"] * c["K"] * 12, "flops": n * c["V"] * 3}
    n = c["G"] * c["W"]
    entries = n * -(-(c["L"] + c["tail"]) // PAGE)
    own_pages = n * (-(-(c["L"] + c["tail"]) // PAGE) - c["L"] // PAGE)
    return {"bytes": entries * 8 + own_pages * 16 + n * 16, "flops": 0}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16)


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def _handle(s, c, **over):
    """The context, head maps and cache description that a user's program keeps."""
    from paper_2605_16928_b200 import binding as rb
    Hkv, n_loc = c.get("Hkv", 1), c.get("n_loc", 0)
    s["rb"], s["ctx"] = rb, rb.Context()
    s["params"] = rb.Params(Hkv * c.get("group", 1), Hkv, [], [], list(range(c.get("n_ih", 0))), list(range(Hkv - n_loc, Hkv)), **over)
    s["cache"] = rb.make_cache(s["k"], s["v"], s.get("ikey"), s["table"], s["lens"])


def prepare(c, seed):
    g = _gen(seed)
    s = dict(case=c, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return {"append": _prepare_append, "chunks": _prepare_chunks, "beam": _prepare_beam, "reorder": _prepare_reorder}[c["kind"]](s, c, g)


def _prepare_append(s, c, g):
    B, T, Hkv, Hq = c["B"], c["T"], c["Hkv"], c["Hkv"] * c["group"]
    new = _parts(T, B)
    lens = [max(n, c["L"] - 777 * b) for b, n in enumerate(new)]
    # the pages that the new tokens lie in; those before them are another program's business here: every entry names some page
    width = -(-max(lens) // PAGE)
    first = [(n - t) // PAGE for n, t in zip(lens, new)]
    own_pages = sum(-(-n // PAGE) - f for n, f in zip(lens, first))
    N = own_pages + 5
    perm = torch.randperm(N, device="cuda", generator=g).int()
    s["table"] = perm[N - 1].expand(B, width).clone()
    at = 0
    for b in range(B):
        n = -(-lens[b] // PAGE) - first[b]
        s["table"][b, first[b]:first[b] + n] = perm[at:at + n]
        at += n
    s["lens"] = _i32(lens)
    s["tok_seq"] = _i32(np.repeat(np.arange(B), new))
    s["tok_pos"] = _i32(np.concatenate([np.arange(n - t, n) for n, t in zip(lens, new)]))
    s["k"], s["v"] = (torch.zeros((N, Hkv, PAGE, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    # one projection makes q, k and v of a token side by side; a few channels of the keys are large
    qkv = _normal(g, T, Hq + 2 * Hkv, DIM)
    qkv[:, Hq:Hq + Hkv, ::29] *= 4
    s["q"], s["kn"], s["vn"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["q_out"] = torch.zeros((T, Hq, DIM), dtype=torch.bfloat16, device="cuda")
    s["freqs"] = 10000.0 ** (-torch.arange(c["rd"] // 2, device="cuda", dtype=torch.float64) * 2 / c["rd"])
    s["ikey"] = s["w_k"] = None
    if c["n_ih"]:
        s["ikey"] = torch.zeros((N, c["n_ih"], PAGE, IDX), dtype=torch.uint8 if c["e4m3"] else torch.bfloat16, device="cuda")
        s["w_k"] = (torch.randn((c["n_ih"], DIM, IDX), device="cuda", generator=g) * DIM ** -0.5).bfloat16()
    if own:
        _handle(s, c)
        s["rope"] = s["rb"].Rope(s["freqs"], rotary_dim=c["rd"], interleaved=c["inter"])
    return s


def _prepare_chunks(s, c, g):
    Hkv, Hq = c["Hkv"], c["Hkv"] * c["group"]
    cs = _chunks(c)
    need = [-(-n // PAGE) for _, n in cs]
    N = sum(need) + 3
    perm = torch.randperm(N, device="cuda", generator=g).int()
    table = torch.full((len(cs), max(need)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(need), device="cuda")[None] < _i32(need)[:, None]] = perm[:sum(need)]
    s["table"], s["lens"] = table, _i32([n for _, n in cs])
    s["k"], s["v"] = _normal(g, N, Hkv, PAGE, DIM), _normal(g, N, Hkv, PAGE, DIM)
    R = sum(r for r, _ in cs)
    s["q"] = _normal(g, R, Hq, DIM)
    s["out"] = torch.zeros((R, Hq, DIM), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((R, Hq), dtype=torch.float32, device="cuda")
    s["seq"] = _i32(range(len(cs)))
    s["start"] = _i32([n - r for r, n in cs])
    s["offsets"] = _i32(np.concatenate([[0], np.cumsum([r for r, _ in cs])]))
    # the plain form takes chunks of similar size together, padded to the longest of them
    alike = {}
    for i, (r, n) in enumerate(cs):
        alike.setdefault((r.bit_length(), n.bit_length()), []).append(i)
    s["alike"] = [(_i32(ids).long(), max(cs[i][0] for i in ids), max(cs[i][1] for i in ids)) for ids in alike.values()]
    if own:
        _handle(s, c, window=c["window"], n_sink=4)
        s["ws"] = torch.empty(s["rb"].rtp_chunk_workspace_bytes(s["params"], len(cs), R), dtype=torch.uint8, device="cuda")
    return s


def _prepare_beam(s, c, g):
    n, V = c["G"] * c["W"], c["V"]
    x = torch.randn((n, V), device="cuda", generator=g) * 3
    x[:, :: max(1, V // 50)] += 6                       # a few likely tokens
    if c["masked"]:
        x[torch.rand((n, V), device="cuda", generator=g) < c["masked"]] = -torch.inf
    s["logits"] = x if c["f32"] else x.bfloat16()
    s["cum"] = -5 * torch.rand(n, device="cuda", generator=g)
    s["finished"] = (torch.rand(n, device="cuda", generator=g) < c["done"]).int()
    K = c["K"]
    s["parent"], s["token"] = (torch.zeros((c["G"], K), dtype=torch.int32, device="cuda") for _ in range(2))
    s["scores"] = torch.zeros((c["G"], K), dtype=torch.float32, device="cuda")
    if own:
        from paper_2605_16928_b200 import binding as rb
        s["rb"], s["ctx"] = rb, rb.Context()
        s["ws"] = torch.empty(rb.rtp_beam_workspace_bytes(n, V, K), dtype=torch.uint8, device="cuda")
    return s


def _prepare_reorder(s, c, g):
    G, W = c["G"], c["W"]
    n = G * W
    L, end = c["L"], c["L"] + c["tail"]
    shared, width = L // PAGE, -(-end // PAGE)
    N = G * shared + n * (width - shared) + 7
    perm = torch.randperm(N, device="cuda", generator=g).int()
    prompt = perm[:G * shared].reshape(G, 1, shared).expand(G, W, shared).reshape(n, shared)
    tail = perm[G * shared:G * shared + n * (width - shared)].reshape(n, width - shared)
    s["table0"] = torch.cat([prompt, tail, torch.full((n, 2), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
    s["refs0"] = torch.zeros(N, dtype=torch.int32, device="cuda")
    s["refs0"].index_add_(0, s["table0"][s["table0"] >= 0].long(), torch.ones(n * width, dtype=torch.int32, device="cuda"))
    s["lens0"] = _i32([end] * n)
    s["table"], s["refs"], s["lens"] = s["table0"].clone(), s["refs0"].clone(), s["lens0"].clone()
    s["src"] = (torch.arange(n, device="cuda") // W * W + torch.randint(0, W, (n,), device="cuda", generator=g)).int()
    s["dst"] = torch.arange(n, device="cuda").int()
    if own:
        s["k"] = s["v"] = torch.zeros((N, 1, PAGE, DIM), dtype=torch.bfloat16, device="cuda")
        _handle(s, c)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if kind == "reorder":   # (the sequences as they were before: surviving hypotheses only would be left after a few passes)
        s["table"].copy_(s["table0"])
        s["refs"].copy_(s["refs0"])
        s["lens"].copy_(s["lens0"])
    if own:
        _run_own(s, kind)
    else:
        {"append": _plain_append, "chunks": _plain_chunks, "beam": _plain_beam, "reorder": _plain_reorder}[kind](s)
    if kind == "append":
        out = dict(q=s["q_out"], k=s["k"], v=s["v"])
        if s["ikey"] is not None:
            out["ikey"] = s["ikey"].view(torch.float8_e4m3fn) if s["case"]["e4m3"] else s["ikey"]
        return out
    if kind == "chunks":
        return dict(out=s["out"], lse=s["lse"])
    if kind == "beam":
        return dict(parent=s["parent"], token=s["token"], scores=s["scores"])
    return dict(table=s["table"], refs=s["refs"], lens=s["lens"])


def _run_own(s, kind):
    rb, ctx = s["rb"], s["ctx"]
    if kind == "append":
        rb.rtp_rope_append(ctx, s["params"], s["cache"], s["rope"], s["q"], s["kn"], s["vn"], s["q_out"], s["w_k"], s["tok_seq"], s["tok_pos"], s["status"])
    elif kind == "chunks":
        rb.rtp_attn_chunks(ctx, s["params"], s["cache"], s["q"], s["seq"], s["start"], s["offsets"],
                           rb.RTP_CHUNK_BY_HEAD if s["case"]["by_head"] else rb.RTP_CHUNK_DENSE, None, s["out"], s["lse"], s["ws"], s["status"])
    elif kind == "beam":
        rb.rtp_beam_select(ctx, s["logits"], s["cum"], s["finished"], 0, s["parent"], s["token"], s["scores"], s["ws"], s["status"])
    else:
        rb.rtp_cache_reorder(ctx, s["params"], s["cache"], s["refs"], s["src"], s["dst"], s["status"])


def _rotate(x, cos, sin, rd, inter):
    """x [T, heads, 128] in 32 bits, cos and sin [T, 1, rd / 2]."""
    r = x[..., :rd]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rd // 2], r[..., rd // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([r, x[..., rd:]], -1)


def _plain_append(s):
    c = s["case"]
    angle = s["tok_pos"].double()[:, None, None] * s["freqs"]       # (a position of 128K times a frequency: 32 bits lose the angle)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    pos = s["tok_pos"].long()
    page = s["table"][s["tok_seq"].long(), pos // PAGE].long()
    s["q_out"].copy_(_rotate(s["q"].float(), cos, sin, c["rd"], c["inter"]))
    s["k"][page, :, pos % PAGE] = _rotate(s["kn"].float(), cos, sin, c["rd"], c["inter"]).bfloat16()
    s["v"][page, :, pos % PAGE] = s["vn"]
    if s["ikey"] is not None:   # (index head j reads KV head j)
        t = torch.matmul(s["kn"][:, :c["n_ih"]].float().transpose(0, 1), s["w_k"].float()).transpose(0, 1)
        s["ikey"][page, :, pos % PAGE] = t.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if c["e4m3"] else t.bfloat16()


def _plain_chunks(s):
    """softmax(q k^T / sqrt(128)) v over the keys that each row sees."""
    c = s["case"]
    Hkv, G, dev = c["Hkv"], c["group"], s["q"].device
    for ids, rows, keys in s["alike"]:
        r, n = torch.arange(rows, device=dev)[None], torch.arange(keys, device=dev)
        off = s["offsets"].long()
        there = r < (off[ids + 1] - off[ids])[:, None]
        at = torch.where(there, off[ids][:, None] + r, off[ids][:, None])
        m = s["start"].long()[ids][:, None] + r                                             # [chunks, rows]
        page = s["table"].long()[ids][:, n // PAGE].clamp(min=0)
        k, v = (s[x][page, :, n % PAGE].transpose(1, 2).float() for x in ("k", "v"))         # [chunks, Hkv, keys, 128]
        v = torch.where((n < s["lens"].long()[ids][:, None])[:, None, :, None], v, 0.0)
        q = s["q"][at].float().reshape(len(ids), rows, Hkv, G, DIM).permute(0, 2, 3, 1, 4).reshape(len(ids), Hkv, G * rows, DIM)
        z = torch.matmul(q, k.transpose(-1, -2)).mul_(DIM ** -0.5).reshape(len(ids), Hkv, G, rows, keys)
        hide = (n > m[..., None])[:, None]                                                  # [chunks, 1, rows, keys]
        if c["by_head"]:
            local = torch.arange(Hkv, device=dev) >= Hkv - c["n_loc"]
            hide = hide | local[None, :, None, None] & (n >= 4) & (n <= m[..., None] - c["window"])[:, None]
        z.masked_fill_(hide[:, :, None], -torch.inf)
        top = z.amax(-1, keepdim=True)
        z.sub_(top).exp_()
        total = z.sum(-1, keepdim=True)
        o = torch.matmul(z.reshape(len(ids), Hkv, G * rows, keys), v).reshape(len(ids), Hkv, G, rows, DIM) / total
        o = o.permute(0, 3, 1, 2, 4).reshape(len(ids), rows, Hkv * G, DIM)
        s["out"][at[there]] = o[there].bfloat16()
        s["lse"][at[there]] = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(len(ids), rows, Hkv * G)[there]


def _plain_beam(s):
    """The best tokens of each beam, equal ones by number, then the best of the group: scores in 64 bits, since neighbours decide."""
    c = s["case"]
    G, W, V, K = c["G"], c["W"], c["V"], c["K"]
    x = s["logits"]
    bits = x.float().view(torch.int32).long()
    order = torch.where(bits < 0, -2147483648 - bits - 1, bits)                            # as the values are ordered
    best = torch.topk(order * 4294967296 + (V - 1 - torch.arange(V, device=x.device)), K).values
    token = V - 1 - best % 4294967296
    d = x.double()
    top = d.amax(-1, keepdim=True).clamp(min=-1e300)
    lse = top + torch.log(torch.exp(d - top).sum(-1, keepdim=True))
    score = s["cum"].double()[:, None] + torch.where(torch.isinf(lse), -torch.inf, torch.gather(d, 1, token) - lse)
    # a beam that has ended stays as it is: one candidate
    ended, first = (s["finished"] != 0)[:, None], torch.arange(K, device=x.device)[None] == 0
    score = torch.where(ended, torch.where(first, s["cum"].double()[:, None], -torch.inf), score)
    token = torch.where(ended, 0, token)
    there = torch.where(ended & ~first, 1, 0).reshape(G, W * K)                            # (places that hold no candidate come last)
    pick = torch.sort(score.reshape(G, W * K), descending=True, stable=True).indices
    pick = torch.gather(pick, 1, torch.sort(torch.gather(there, 1, pick), stable=True).indices)[:, :K]
    some = torch.gather(there, 1, pick) == 0
    s["scores"].copy_(torch.where(some, torch.gather(score.reshape(G, W * K), 1, pick), -torch.inf))
    s["parent"].copy_(torch.where(some, pick // K + W * torch.arange(G, device=x.device)[:, None], -1))
    s["token"].copy_(torch.where(some, torch.gather(token.reshape(G, W * K), 1, pick), -1))


def _plain_reorder(s):
    table, refs, src, dst = s["table"], s["refs"], s["src"].long(), s["dst"].long()
    old, new = table[dst], table[src]
    refs.index_add_(0, old.clamp(min=0).reshape(-1).long(), -(old >= 0).reshape(-1).int())
    refs.index_add_(0, new.clamp(min=0).reshape(-1).long(), (new >= 0).reshape(-1).int())
    table[dst] = new
    s["lens"][dst] = s["lens"][src]


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(c, seed):
    if c["kind"] == "reorder":
        return None
    s = prepare(c, seed)
    return {"append": _exact_append, "chunks": _exact_chunks, "beam": _exact_beam}[c["kind"]](s, c)


def _exact_append(s, c):
    rd, T = c["rd"], c["T"]
    th = torch.outer(s["tok_pos"].double(), s["freqs"])
    turn = torch.polar(torch.ones_like(th), th)                                            # e^(i angle)

    def rot(x):
        y = x.double().clone()
        for i in range(rd // 2):
            a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + rd // 2)
            w = torch.complex(y[..., a], y[..., b]) * turn[:, i:i + 1]
            y[..., a], y[..., b] = w.real, w.imag
        return y

    pos = s["tok_pos"].long()
    page, slot = s["table"].long()[s["tok_seq"].long(), pos // PAGE], pos % PAGE
    k, v = s["k"].double(), s["v"].double()
    k[page, :, slot], v[page, :, slot] = rot(s["kn"]), s["vn"].double()
    out = dict(q=rot(s["q"]), k=k, v=v)
    if c["n_ih"]:
        ik = torch.zeros(s["ikey"].shape, dtype=torch.float64, device="cuda")
        for j in range(c["n_ih"]):
            ik[page, j, slot] = s["kn"][:, j].double() @ s["w_k"][j].double()
        out["ikey"] = ik
    return out


def _exact_chunks(s, c):
    out, lse = s["out"].double(), s["lse"].double()
    off = s["offsets"].tolist()
    for i, (r, n) in enumerate(_chunks(c)):
        t = torch.arange(n, device="cuda")
        p, o = s["table"][i].long()[t // PAGE], t % PAGE
        m = torch.arange(n - r, n, device="cuda")[:, None]
        for h in range(c["Hkv"] * c["group"]):
            j = h // c["group"]
            see = t <= m
            if c["by_head"] and j >= c["Hkv"] - c["n_loc"]:
                see &= (t < 4) | (t > m - c["window"])
            z = s["q"][off[i]:off[i] + r, h].double() @ s["k"][p, j, o].double().T / math.sqrt(DIM)
            z[~see] = -math.inf
            l = torch.logsumexp(z, -1)
            out[off[i]:off[i] + r, h] = torch.exp(z - l[:, None]) @ s["v"][p, j, o].double()
            lse[off[i]:off[i] + r, h] = l
    return dict(out=out, lse=lse)


def _exact_beam(s, c):
    G, W, V, K = c["G"], c["W"], c["V"], c["K"]
    best = torch.full((G, K), -math.inf, dtype=torch.float64, device="cuda")
    for g in range(G):
        rows = []
        for b in range(g * W, g * W + W):
            if int(s["finished"][b]):
                rows.append(s["cum"][b:b + 1].double())
            else:
                x = s["logits"][b].double()
                rows.append(torch.topk(s["cum"][b].double() + x - torch.logsumexp(x, 0), min(K, V)).values)
        v = torch.sort(torch.cat(rows), descending=True).values[:K]
        best[g, :len(v)] = v
    return dict(parent=None, token=None, scores=best)
