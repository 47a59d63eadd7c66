"""Measured cases of the 4-bit K/V cache and of the page operations.

Operators:
  prompt    K/V rows quantised into a 4-bit cache and pages of it expanded to bf16 (``rtp_kv_append``, ``rtp_kv_expand``)
  dense, local, list, pages
            decode attention over a 4-bit cache: the whole prefix, sink + window, token lists, page lists
            (``rtp_dense_attn_decode``, ``rtp_local_attn``, ``rtp_sparse_attn_decode``, ``rtp_sparse_attn_decode_blocks``)
  resample  earlier samples of a prompt are freed, new ones forked from it and given room for their next tokens
            (``rtp_cache_free``, ``rtp_cache_fork``, ``rtp_cache_reserve``)
  copy, compact
            pages copied; used pages moved to the front of the pool (``rtp_cache_copy_pages``, ``rtp_cache_compact``)

The 4-bit cache: a group of 16 channels of a token has a scale, an unsigned 8-bit float with 5 exponent and 3 mantissa bits
(bias 15; scale = amax / 6 rounded to nearest even, at most 10240), and 16 codes E2M1 (sign, 2 exponent bits, 1 mantissa bit:
0, .5, 1, 1.5, 2, 3, 4, 6), value / scale rounded to nearest even.  k_pages / v_pages: uint8 [pages, KV heads, 64, 64], channel
2 b in the low half of byte b; kv_scales: uint8 [pages, KV heads, 64, 16], the 8 scales of K, then those of V.
"""
import numpy as np
import torch

own = False

PAGE, DIM = 64, 128
MAX_SCALE = 10240.0


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decode step of a batch of eight: the newest K/V rows go into the cache, their pages are read back
        dict(name="prompt_step_b8", kind="prompt", B=8, T=1, L=32768, Hkv=8, group=4, whole=False),
        # a chunk of 8192 prompt tokens appended behind 120K others, the whole 128K prefix expanded for the prefill attention
        dict(name="prompt_chunk_8k_of_128k", kind="prompt", B=1, T=8192, L=131072, Hkv=8, group=4, whole=True),
        # one short conversation
        dict(name="dense_b1_4k", kind="dense", B=1, L=4096, Hkv=8, group=4),
        # long contexts, every head over everything: the dense comparator of the decode sweep
        dict(name="dense_b4_512k", kind="dense", B=4, L=524288, Hkv=8, group=4),
        # local heads of a batch of sixteen: 4 sinks and 4096 recent tokens on six of eight KV heads
        dict(name="local_b16_w4096", kind="local", B=16, L=32768, Hkv=8, group=4, n_loc=6, window=4096, n_sink=4),
        # retrieval heads of a batched decode: about 5 % of 32K tokens in a list per query head, two retrieval KV heads
        dict(name="list_b8_32k", kind="list", B=8, L=32768, Hkv=8, group=4, n_kv_ret=2, S=1639),
        # retrieval heads at 512K, a tenth of the tokens selected
        dict(name="list_b4_512k", kind="list", B=4, L=524288, Hkv=8, group=4, n_kv_ret=2, S=52429),
        # the same with whole pages selected, a fifth of them
        dict(name="pages_b4_512k", kind="pages", B=4, L=524288, Hkv=8, group=4, n_kv_ret=2, S=1639),
        # eight samples branching from one prompt of about 4K tokens
        dict(name="resample_8_of_4k", kind="resample", n=8, parents=1, L=4099, add=1, Hkv=8, n_ih=2, spare=100),
        # 64 samples branching from four prompts of about 32K tokens, room for a block of 200 tokens each
        dict(name="resample_64_of_32k", kind="resample", n=64, parents=4, L=32803, add=200, Hkv=8, n_ih=2, spare=1000),
        # a prompt of 16K tokens copied page by page
        dict(name="copy_256_pages", kind="copy", n=256, N=1024, Hkv=8, n_ih=2),
        # a pool of 16K pages, half of it in use, 3001 pages above the others moved down
        dict(name="compact_16k_pages", kind="compact", B=16, N=16384, U=8192, M=3001, Hkv=8, n_ih=2),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["prompt", "dense", "local", "list", "pages", "resample", "copy", "compact"])
    Hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
    if kind == "prompt":
        L = _log(rng, 1, 131072)
        return dict(kind=kind, B=rng.randint(1, 4), T=min(L, _log(rng, 1, 8192)), L=L, Hkv=Hkv, group=group, whole=rng.random() < 0.5)
    if kind in ("resample", "copy", "compact"):
        n_ih = rng.randint(0, 2)
        if kind == "resample":
            parents = rng.randint(1, 4)
            return dict(kind=kind, n=_log(rng, 1, 64), parents=parents, L=_log(rng, 200, 32768), add=_log(rng, 1, 200), Hkv=Hkv, n_ih=n_ih,
                        spare=_log(rng, 1, 2000))
        if kind == "copy":
            n = _log(rng, 1, 1000)
            return dict(kind=kind, n=n, N=2 * n + _log(rng, 1, 1000), Hkv=Hkv, n_ih=n_ih)
        N = _log(rng, 64, 16384)
        U = rng.randint(1, N)
        return dict(kind=kind, B=rng.randint(1, 16), N=N, U=U, M=rng.randint(0, min(U, N - U)), Hkv=Hkv, n_ih=n_ih)
    L = _log(rng, 1, 524288)
    B = rng.randint(1, max(1, min(16, 2097152 // L)))
    c = dict(kind=kind, B=B, L=L, Hkv=Hkv, group=group)
    if kind == "local":
        c.update(n_loc=rng.randint(1, Hkv), window=_log(rng, 1, 8192), n_sink=rng.randint(0, 70))
    if kind == "list":
        c.update(n_kv_ret=rng.randint(1, min(2, Hkv)), S=max(1, int(L * 10 ** rng.uniform(-3, -0.7))))
    if kind == "pages":
        c.update(n_kv_ret=rng.randint(1, min(2, Hkv)), S=max(1, int(-(-L // PAGE) * 10 ** rng.uniform(-2, -0.7))))
    return c


def _lens(c):
    """Lengths of the batch's sequences: ragged, the first one the longest."""
    return [c["L"] - (b * 1009) % (c["L"] // 4 + 1) for b in range(c["B"])]


def _counts(c, n_units):
    """Entries of the lists, (row, head) by (row, head): between half of S and S, never more than the row has."""
    lens = _lens(c)
    most = [-(-n // PAGE) if c["kind"] == "pages" else n for n in lens]
    return [[min(max(1, c["S"] - (97 * (b * n_units + u)) % (c["S"] // 2 + 1)), most[b]) for u in range(n_units)] for b in range(c["B"])]


def work(c):
    kind = c["kind"]
    Hkv = c["Hkv"]
    if kind == "prompt":
        lens = [c["L"]] * c["B"]
        pages = sum(-(-n // PAGE) if c["whole"] else -(-n // PAGE) - (n - c["T"]) // PAGE for n in lens)
        rows = c["B"] * c["T"]
        return {"bytes": rows * Hkv * (512 + 144) + pages * Hkv * PAGE * (144 + 512), "flops": rows * Hkv * 256 * 4 + pages * Hkv * PAGE * 256}
    if kind in ("copy", "compact", "resample"):
        page = 2 * Hkv * PAGE * DIM * 2 + c["n_ih"] * PAGE * 16 * 2
        if kind == "copy":
            return {"bytes": 2 * c["n"] * page + 8 * c["n"], "flops": 0}
        if kind == "compact":
            return {"bytes": 2 * c["M"] * page + 8 * c["N"] + 8 * c["U"], "flops": 0}
        lens = _parent_lens(c)
        moved, entries = 0, 0
        for j in range(c["n"]):
            ln = lens[j % c["parents"]]
            moved += 1 if ln % PAGE else 0
            entries += -(-(ln + c["add"]) // PAGE)
        return {"bytes": 2 * moved * page + entries * 4 * 4 + 8 * _pool(c), "flops": 0}
    lens = _lens(c)
    G = c["group"]
    io = c["B"] * Hkv * G * (512 + 4)
    if kind == "dense":
        toks = sum(lens) * Hkv
        heads = toks * G
    elif kind == "local":
        toks = sum(min(n, c["n_sink"] + min(c["window"], max(0, n - c["n_sink"]))) for n in lens) * c["n_loc"]
        heads = toks * G
    else:   # a KV head has to supply the union of its query heads' lists, drawn independently of one another
        toks = heads = 0
        for n, cnt in zip(lens, _counts(c, c["n_kv_ret"] * G)):
            size = [min(n, x * PAGE) if kind == "pages" else x for x in cnt]
            heads += sum(size)
            for k in range(c["n_kv_ret"]):
                out = 1.0
                for x in size[k * G:(k + 1) * G]:
                    out *= 1.0 - x / n
                toks += int(n * (1.0 - out))
    return {"bytes": toks * 144 + io, "flops": heads * 4 * DIM}


# ---------------------------------------------------------------------------------------------- the format, in 32 bits
def _scale_values(dev, dtype=torch.float32):
    u = torch.arange(256, device=dev)
    e, m = (u >> 3).to(dtype), (u & 7).to(dtype)
    return torch.where(e == 0, m * 2.0 ** -17, (1.0 + m / 8) * torch.exp2(e - 15))


def _code_values(dev, dtype=torch.float32):
    """The two values of each byte: [256, 2]."""
    v = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=dev, dtype=dtype)
    v = torch.cat([v, -v])
    u = torch.arange(256, device=dev)
    return torch.stack([v[u & 15], v[u >> 4]], -1)


def _quantise(x):
    """x [..., 128] -> codes uint8 [..., 64], scales uint8 [..., 8]."""
    x = x.float().unflatten(-1, (8, 16))
    t = (x.abs().amax(-1, keepdim=True) / 6.0).clamp(max=MAX_SCALE)
    e = (torch.frexp(t).exponent - 1).clamp(min=-14)
    m = torch.round(torch.ldexp(t, 3 - e))                      # 8 .. 16, below 8 for subnormal scales
    s = torch.ldexp(m, e - 3)
    scale = ((e + 14) * 8 + m.int()).to(torch.uint8)             # (m = 16 carries into the exponent)
    a = torch.where(s > 0, x / s, torch.zeros_like(x))
    mag = a.abs().clamp(max=6.0)
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    r = torch.round(mag / step) * step
    code = torch.where(r <= 2, r * 2, torch.where(r <= 4, r + 2, r / 2 + 4)).int()
    code = code + 8 * (a < 0).int()
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.squeeze(-1)


def _dequantise(codes, scales):
    """codes uint8 [..., 64], scales uint8 [..., 8] -> fp32 [..., 128]."""
    v = torch.index_select(_code_values(codes.device), 0, codes.reshape(-1).int()).reshape(*codes.shape[:-1], 8, 16)
    s = torch.index_select(_scale_values(codes.device), 0, scales.reshape(-1).int()).reshape(*scales.shape, 1)
    return v.mul_(s).flatten(-2)


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _handle(s, c, n_loc=(), n_ret_kv=0, **over):
    """The context, head maps and cache description that a user's program keeps."""
    from paper_2605_16928_b200 import binding as rb
    Hkv, G = c["Hkv"], c.get("group", 1)
    ret = list(range(n_ret_kv * G))
    s["rb"], s["ctx"] = rb, rb.Context()
    index_kv = [i % Hkv for i in range(max(n_ret_kv, c.get("n_ih", 0)))]
    s["params"] = rb.Params(Hkv * G, Hkv, ret, [i // G for i in ret], index_kv, list(n_loc), **over)
    s["cache"] = rb.make_cache(s["k"], s["v"], s.get("ikey"), s["table"], s["lens"], kv_scales=s.get("scales"))
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")


def _cache4(B, L, Hkv, g):
    """A 4-bit cache of B sequences: keys with a few large channels, values, both N(0, 1) otherwise, quantised."""
    nP = -(-L // PAGE)
    N = B * nP + 3
    k = torch.zeros((N, Hkv, PAGE, DIM // 2), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    sc = torch.zeros((N, Hkv, PAGE, 16), dtype=torch.uint8, device="cuda")
    gain = torch.ones((Hkv, 1, DIM), device="cuda")
    gain[..., ::29] = 4.0
    for lo in range(0, N, 2048):
        hi = min(N, lo + 2048)
        k[lo:hi], sc[lo:hi, ..., :8] = _quantise((torch.randn((hi - lo, Hkv, PAGE, DIM), device="cuda", generator=g) * gain).bfloat16())
        v[lo:hi], sc[lo:hi, ..., 8:] = _quantise(torch.randn((hi - lo, Hkv, PAGE, DIM), device="cuda", generator=g).bfloat16())
    table = torch.randperm(N, device="cuda", generator=g)[:B * nP].reshape(B, nP).int().contiguous()
    return dict(k=k, v=v, scales=sc, table=table)


def prepare(c, seed):
    g = _gen(seed)
    kind = c["kind"]
    if kind in ("copy", "compact", "resample"):
        return _prepare_pages(c, g)
    B, L, Hkv = c["B"], c["L"], c["Hkv"]
    s = dict(case=c, **_cache4(B, L, Hkv, g))
    lens = [L] * B if kind == "prompt" else _lens(c)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if kind == "prompt":
        T = c["T"]
        s["k_new"], s["v_new"] = (torch.randn((B * T, Hkv, DIM), device="cuda", generator=g).bfloat16() for _ in range(2))
        s["tok_seq"] = torch.arange(B, device="cuda").repeat_interleave(T).int()
        s["tok_pos"] = (L - T + torch.arange(T, device="cuda")).repeat(B).int()
        s["pages"] = s["table"][:, 0 if c["whole"] else (L - T) // PAGE:].reshape(-1).contiguous()
        n = s["pages"].numel()
        s["k_out"], s["v_out"] = (torch.zeros((n, Hkv, PAGE, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        if own:
            _handle(s, c)
        return s
    G = c["group"]
    Hq = Hkv * G
    s["q"] = torch.randn((B, Hq, DIM), device="cuda", generator=g).bfloat16()
    s["row_seq"] = torch.arange(B, device="cuda").int()
    s["row_pos"] = s["lens"] - 1
    s["out"] = torch.zeros((B, Hq, DIM), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros((B, Hq), dtype=torch.float32, device="cuda")
    n_loc, n_ret, over = [], 0, {}
    if kind == "local":
        n_loc, over = list(range(Hkv - c["n_loc"], Hkv)), dict(window=c["window"], n_sink=c["n_sink"])
    if kind in ("list", "pages"):
        n_ret = c["n_kv_ret"]
        cnt = _counts(c, n_ret * G)
        s["cnt"] = torch.tensor(cnt, dtype=torch.int32, device="cuda")
        stride = max(max(x) for x in cnt)
        most = (s["lens"] if kind == "list" else (s["lens"] + PAGE - 1) // PAGE)[:, None, None]
        # one entry from each of cnt equal parts of the row, ascending
        i = torch.arange(stride, device="cuda")[None, None]
        lo = i * most // s["cnt"][..., None]
        hi = (i + 1) * most // s["cnt"][..., None]
        r = torch.rand((B, n_ret * G, stride), device="cuda", generator=g, dtype=torch.float64)
        s["idx"] = torch.minimum(lo + (r * (hi - lo)).long(), most - 1).int().contiguous()
    if own:
        _handle(s, c, n_loc, n_ret, **over)
        rows = s["rb"].rtp_workspace_bytes(s["params"], B, L)
        s["ws"] = torch.empty(max(rows, 1 << 20), dtype=torch.uint8, device="cuda")
    return s


def _parent_lens(c):
    return [max(1, c["L"] - 1000 * i) for i in range(c["parents"])]


def _pool(c):
    lens = _parent_lens(c)
    return sum(-(-n // PAGE) for n in lens) + c["n"] * (2 + c["add"] // PAGE) + c["spare"]


def _prepare_pages(c, g):
    kind, Hkv, n_ih = c["kind"], c["Hkv"], c["n_ih"]
    N = _pool(c) if kind == "resample" else c["N"]
    s = dict(case=c)
    s["k"], s["v"] = (torch.randn((N, Hkv, PAGE, DIM), device="cuda", generator=g, dtype=torch.bfloat16) for _ in range(2))
    s["ikey"] = torch.randn((N, n_ih, PAGE, 16), device="cuda", generator=g, dtype=torch.bfloat16) if n_ih else None
    perm = torch.randperm(N, device="cuda", generator=g)
    s["refs"] = torch.zeros(N, dtype=torch.int32, device="cuda")
    if kind == "copy":
        s["src"], s["dst"] = perm[:c["n"]].int().contiguous(), perm[c["n"]:2 * c["n"]].int().contiguous()
        s["table"], s["lens"] = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    elif kind == "resample":
        lens = _parent_lens(c)
        P = c["parents"]
        used = [-(-n // PAGE) for n in lens]
        width = -(-(max(lens) + c["add"]) // PAGE) + 1
        s["table"] = torch.full((P + c["n"], width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(used):
            s["table"][i, :n] = perm[at:at + n].int()
            at += n
        s["refs"][perm[:at]] = 1
        s["lens"] = torch.tensor(lens + [0] * c["n"], dtype=torch.int32, device="cuda")
        order = torch.randperm(c["n"], device="cuda", generator=g)
        s["src"] = (order % P).int()
        s["dst"] = (P + torch.arange(c["n"], device="cuda")).int()
        s["add"] = torch.full((c["n"],), c["add"], dtype=torch.int32, device="cuda")
    else:
        U, M, B = c["U"], c["M"], c["B"]
        low = torch.randperm(U, device="cuda", generator=g)[:U - M]
        high = U + torch.randperm(N - U, device="cuda", generator=g)[:M]
        ids = torch.cat([low, high])[torch.randperm(U, device="cuda", generator=g)]
        s["refs"][ids] = 1
        width = -(-U // B)
        s["table"] = torch.full((B * width,), -1, dtype=torch.int32, device="cuda")
        s["table"][:U] = ids.int()
        s["table"] = s["table"].reshape(B, width).contiguous()
        s["lens"] = ((s["table"] >= 0).sum(1) * PAGE).int()
        s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
        s["n_used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        _handle(s, c)
        n = s["rb"].rtp_cache_workspace_bytes(s["cache"], c.get("n", c.get("B")))
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _page_outputs(s):
    out = dict(k=s["k"], v=s["v"])
    if s["ikey"] is not None:
        out["ikey"] = s["ikey"]
    if s["case"]["kind"] != "copy":
        out.update(table=s["table"], refs=s["refs"], lens=s["lens"])
    if s["case"]["kind"] == "compact":
        out.update(n_used=s["n_used"])
    return out


def _run_own(s):
    rb, ctx, p, cache, status = s["rb"], s["ctx"], s["params"], s["cache"], s["status"]
    kind = s["case"]["kind"]
    if kind == "prompt":
        rb.rtp_kv_append(ctx, p, cache, s["k_new"], s["v_new"], s["tok_seq"], s["tok_pos"], status)
        rb.rtp_kv_expand(ctx, p, cache, s["pages"], None, s["k_out"], s["v_out"], status)
        return dict(k=s["k_out"], v=s["v_out"])
    if kind == "copy":
        rb.rtp_cache_copy_pages(ctx, p, cache, s["src"], s["dst"], status)
        return _page_outputs(s)
    if kind == "resample":
        rb.rtp_cache_free(ctx, p, cache, s["refs"], s["dst"], status)
        rb.rtp_cache_fork(ctx, p, cache, s["refs"], s["src"], s["dst"], status)
        rb.rtp_cache_reserve(ctx, p, cache, s["refs"], s["dst"], s["add"], s["ws"], status)
        return _page_outputs(s)
    if kind == "compact":
        s["table"].copy_(s["table0"])   # (the pool as it was before: a pass leaves the moved pages' old places as they are)
        s["refs"].copy_(s["refs0"])
        rb.rtp_cache_compact(ctx, p, cache, s["refs"], s["n_used"], s["ws"], status)
        return _page_outputs(s)
    args = (ctx, p, cache, s["q"], s["row_seq"], s["row_pos"])
    if kind == "dense":
        rb.rtp_dense_attn_decode(*args, None, s["out"], s["lse"], s["ws"], status)
    elif kind == "local":
        rb.rtp_local_attn(*args, 0, 0, s["case"]["B"], s["out"], s["lse"], s["ws"], status)
    elif kind == "list":
        rb.rtp_sparse_attn_decode(*args, s["idx"], s["cnt"], s["out"], s["lse"], s["ws"], status)
    else:
        rb.rtp_sparse_attn_decode_blocks(*args, s["idx"], s["cnt"], s["out"], s["lse"], s["ws"], status)
    return dict(out=s["out"], lse=s["lse"])


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "prompt":
        phys = s["table"][s["tok_seq"].long(), s["tok_pos"].long() // PAGE].long()
        off = s["tok_pos"].long() % PAGE
        kc, ks = _quantise(s["k_new"])
        vc, vs = _quantise(s["v_new"])
        s["k"][phys, :, off], s["v"][phys, :, off] = kc, vc
        s["scales"][phys, :, off] = torch.cat([ks, vs], -1)
        ids = s["pages"].long()
        sc = s["scales"][ids]
        return dict(k=_dequantise(s["k"][ids], sc[..., :8]).bfloat16(), v=_dequantise(s["v"][ids], sc[..., 8:]).bfloat16())
    if kind == "copy":
        _plain_move(s, s["src"].long(), s["dst"].long())
        return _page_outputs(s)
    if kind == "resample":
        return _plain_resample(s)
    if kind == "compact":
        return _plain_compact(s)
    return _plain_attention(s)


def _plain_attention(s):
    """softmax(q k^T / sqrt(128)) v over the tokens that each unit (a KV head with its group, or a query head) sees."""
    c = s["case"]
    kind, B, Hkv, G = c["kind"], c["B"], c["Hkv"], c["group"]
    dev = s["q"].device
    lens = s["lens"].long()[:, None, None]
    if kind == "dense":
        units, per = torch.arange(Hkv, device=dev), G
        tok = torch.arange(c["L"], device=dev)[None, None].expand(B, 1, -1)
        ok = tok < lens
    elif kind == "local":
        units, per = torch.arange(Hkv - c["n_loc"], Hkv, device=dev), G
        sink = torch.arange(c["n_sink"], device=dev)[None, None].expand(B, 1, -1)
        tok = torch.cat([sink, lens - c["window"] + torch.arange(c["window"], device=dev)], -1)
        ok = torch.cat([sink < lens, tok[..., c["n_sink"]:] >= c["n_sink"]], -1)
        tok = tok.clamp(min=0)
    else:
        units, per = torch.arange(c["n_kv_ret"] * G, device=dev) // G, 1
        tok = s["idx"].long()
        ok = torch.arange(tok.shape[-1], device=dev) < s["cnt"][..., None]
        if kind == "pages":
            tok = (tok[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(-2)
            ok = ok.repeat_interleave(PAGE, -1) & (tok < lens)
    tok = torch.minimum(tok, lens - 1)
    phys = s["table"].long()[torch.arange(B, device=dev)[:, None, None], tok // PAGE]
    at = (phys, units[None, :, None], tok % PAGE)
    first = int(c["Hkv"] - c["n_loc"]) * G if kind == "local" else 0
    q = s["q"].float()[:, first:first + units.numel() * per].reshape(B, units.numel(), per, DIM)
    sc = s["scales"][at]
    logit = torch.matmul(q, _dequantise(s["k"][at], sc[..., :8]).transpose(-1, -2)) * DIM ** -0.5
    logit = torch.where(ok[:, :, None], logit, -torch.inf)
    m = logit.amax(-1, keepdim=True)
    e = torch.exp(logit - m)
    z = e.sum(-1, keepdim=True)
    o = torch.matmul(e, _dequantise(s["v"][at], sc[..., 8:])) / z
    s["out"][:, first:first + units.numel() * per] = o.reshape(B, -1, DIM).bfloat16()
    s["lse"][:, first:first + units.numel() * per] = (m + torch.log(z)).reshape(B, -1)
    return dict(out=s["out"], lse=s["lse"])


def _plain_move(s, src, dst):
    s["k"][dst], s["v"][dst] = s["k"][src], s["v"][src]
    if s["ikey"] is not None:
        s["ikey"][dst] = s["ikey"][src]


def _plain_resample(s):
    table, refs, lens, dev = s["table"], s["refs"], s["lens"], s["refs"].device
    src, dst, add = s["src"].long(), s["dst"].long(), s["add"].long()
    N, W = refs.numel(), table.shape[1]
    # free
    old = table[dst]
    refs.index_add_(0, old.clamp(min=0).reshape(-1).long(), -(old >= 0).reshape(-1).int())
    table[dst] = -1
    # fork
    ln = lens[src].long()
    have = (ln + PAGE - 1) // PAGE
    page = torch.arange(W, device=dev)
    shared = page < have[:, None]
    table[dst] = torch.where(shared, table[src], -1)
    refs.index_add_(0, table[dst].clamp(min=0).reshape(-1).long(), shared.reshape(-1).int())
    lens[dst] = lens[src]
    # room for the next tokens: copies of shared pages that are going to be written, and new pages, the lowest free ones in order
    part = (ln % PAGE > 0) & (add > 0)
    last = torch.where(part, table[dst, ln // PAGE].long(), -1)
    earlier = ((last[:, None] == last[None]) & torch.ones((len(src),) * 2, dtype=torch.bool, device=dev).tril(-1)).sum(1)
    cow = part & (refs[last.clamp(min=0)] - earlier > 1)
    want = (page >= have[:, None]) & (page < ((ln + add + PAGE - 1) // PAGE)[:, None]) | (cow[:, None] & (page == (ln // PAGE)[:, None]))
    free = torch.argsort((refs != 0).int(), stable=True)
    rank = (want.reshape(-1).cumsum(0) - 1).clamp(min=0).reshape(want.shape)
    new = free[rank]
    refs.index_add_(0, last.clamp(min=0), -cow.int())
    refs.index_add_(0, torch.where(want, new, 0).reshape(-1), want.reshape(-1).int())
    table[dst] = torch.where(want, new.int(), table[dst])
    i = cow.nonzero()[:, 0]
    _plain_move(s, last[i], table[dst[i], ln[i] // PAGE].long())
    return _page_outputs(s)


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    table.copy_(s["table0"])
    refs.copy_(s["refs0"])
    used = refs > 0
    n = used.sum()
    ids = torch.arange(refs.numel(), device=refs.device)
    src, dst = (used & (ids >= n)).nonzero()[:, 0], (~used & (ids < n)).nonzero()[:, 0]
    to = ids.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    refs[dst] = refs[src]
    refs[src] = 0
    _plain_move(s, src, dst)
    s["n_used"].copy_(n)
    return _page_outputs(s)


# ---------------------------------------------------------------------------------------------- in 64 bits
def _nearest_even(x, grid):
    """The index of the value of an ascending grid that is next to x >= 0; halfway, the even one."""
    hi = torch.searchsorted(grid, x).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - x, x - grid[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_values(x):
    """What the format holds of x [..., 128], in 64 bits."""
    scales = torch.tensor([m / 8 * 2.0 ** -14 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-14, 14) for m in range(8)],
                          dtype=torch.float64, device=x.device)
    scales = scales[scales <= MAX_SCALE]
    g = x.double().reshape(*x.shape[:-1], 8, 16)
    s = scales[_nearest_even(g.abs().amax(-1) / 6, scales)][..., None]
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    r = torch.where(s == 0, 0.0, g.abs() / torch.where(s == 0, 1.0, s))
    return (torch.sign(g) * grid[_nearest_even(r, grid)] * s).reshape(x.shape)


def _exact_read(codes, scales):
    """codes uint8 [n, 64], scales uint8 [n, 8] -> float64 [n, 128]."""
    v = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=torch.float64, device=codes.device)
    x = torch.stack([v[(codes & 15).long()], v[(codes >> 4).long()]], -1).reshape(-1, 8, 16)
    e, m = (scales >> 3).long(), (scales & 7).double()
    f = torch.where(e > 0, 8 + m, m) * 2.0 ** (torch.maximum(e, torch.ones_like(e)) - 18).double()
    return (x * f[..., None]).reshape(-1, DIM)


def exact(c, seed):
    kind = c["kind"]
    if kind in ("copy", "compact", "resample"):
        return None
    s = prepare(c, seed)
    if kind == "prompt":
        outs = {}
        for name, pages, new, at in (("k", s["k"], s["k_new"], 0), ("v", s["v"], s["v_new"], 8)):
            ids = s["pages"].long()
            vals = _exact_read(pages[ids].reshape(-1, 64), s["scales"][ids][..., at:at + 8].reshape(-1, 8)).reshape(len(ids), c["Hkv"], PAGE, DIM)
            place = torch.full((pages.shape[0],), -1, device="cuda")
            place[ids] = torch.arange(len(ids), device="cuda")
            pos = s["tok_pos"].long()
            vals[place[s["table"][s["tok_seq"].long(), pos // PAGE].long()], :, pos % PAGE] = _exact_values(new)
            outs[name] = vals
        return outs
    out, lse = s["out"].double(), s["lse"].double()
    G = c["group"]
    for b, n in enumerate(_lens(c)):
        groups = [(h, list(range(h * G, h * G + G)), None) for h in range(c["Hkv"])]
        if kind == "local":
            seen = sorted(set(range(min(n, c["n_sink"]))) | set(range(max(0, n - c["window"]), n)))
            groups = [(h, hs, torch.tensor(seen, device="cuda")) for h, hs, _ in groups[c["Hkv"] - c["n_loc"]:]]
        if kind in ("list", "pages"):
            groups = []
            for i in range(c["n_kv_ret"] * G):
                t = s["idx"][b, i, :int(s["cnt"][b, i])].long()
                if kind == "pages":
                    t = (t[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)
                    t = t[t < n]
                groups.append((i // G, [i], t))
        for h, heads, t in groups:
            t = torch.arange(n, device="cuda") if t is None else t
            p, o = s["table"][b].long()[t // PAGE], t % PAGE
            sc = s["scales"][p, h, o]
            z = s["q"][b, heads].double() @ _exact_read(s["k"][p, h, o], sc[:, :8]).T / np.sqrt(DIM)
            l = torch.logsumexp(z, -1)
            out[b, heads] = torch.exp(z - l[:, None]) @ _exact_read(s["v"][p, h, o], sc[:, 8:])
            lse[b, heads] = l
    return dict(out=out, lse=lse)
