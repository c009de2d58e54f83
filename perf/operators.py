"""Cases for the operators that serve from a paged KV cache between two topology switches: writing new tokens into a cache
held in 4 bits (norm, rotation and quantisation in one pass) and reading them back, attention over that cache, and the
management of its pages (fork, free, compact, copy).

Where `own` is false, `run` computes an operator from elementary torch operations in 32 bits; where it is true, it makes
the calls of the package.
"""
import math

import torch

own = False

GROUP = 64   # dims that share a scale and a minimum
TILE = 16    # tokens whose codes lie together, followed by their scales and minima
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # The tiny shape's heads, one new token for each of 8 short sequences: nothing but latency.
        {"name": "append_tiny", "op": "append", "q_heads": 4, "kv_heads": 4, "head_dim": 64, "block_size": 16, "dtype": "f16",
         "seqs": 8, "new": 1, "past": 200, "ragged": True, "norm": False, "rotary": 32, "interleaved": True},
        # One decode step of a full batch on the 70B shape.
        {"name": "append_decode_70b", "op": "append", "q_heads": 64, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 256, "new": 1, "past": 2048, "ragged": True, "norm": False, "rotary": 128, "interleaved": False},
        # Prompts of uneven lengths written in one go, heads of the 30B-A3B shape with its norms of queries and keys.
        {"name": "append_prompts_30b", "op": "append", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 11, "new": 2900, "past": 0, "ragged": True, "norm": True, "rotary": 128, "interleaved": False},
        # The tiny shape, lengths in [1, 256], one query each: latency.
        {"name": "attend_tiny", "op": "attend", "q_heads": 4, "kv_heads": 4, "head_dim": 64, "block_size": 16, "dtype": "f16",
         "seqs": 8, "queries": 1, "length": 128, "spread": "uniform", "window": 0, "lse": False},
        # A decode step over the 70B shape's long-context lognormal lengths, about 100 thousand cached tokens, with the
        # logarithms of the sums that merge partial results of ranks.
        {"name": "attend_decode_70b", "op": "attend", "q_heads": 64, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 29, "queries": 1, "length": 3400, "spread": "lognormal", "window": 0, "lse": True},
        # The edge stress: 2048 sequences of 1 to 63 tokens in blocks of 32, one rank of TP2.
        {"name": "attend_stress", "op": "attend", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 32, "dtype": "bf16",
         "seqs": 2048, "queries": 1, "length": 32, "spread": "uniform", "window": 0, "lse": False},
        # One very long sequence on the 32B shape (five query heads for each KV head).
        {"name": "attend_long_32b", "op": "attend", "q_heads": 40, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 1, "queries": 1, "length": 131071, "spread": "fixed", "window": 0, "lse": True},
        # Chunks of two prompts that follow cached text, 30B-A3B heads.
        {"name": "attend_prompt_30b", "op": "attend", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 2, "queries": 2048, "length": 8191, "spread": "fixed", "window": 0, "lse": False},
        # Two continuations for each of 4 sequences of the tiny shape.
        {"name": "fork_tiny", "op": "fork", "layers": 2, "heads": 4, "head_dim": 64, "block_size": 16, "elem_bytes": 2,
         "seqs": 4, "children": 2, "length": 100},
        # Seven more samples for each of 64 prompts, one pipeline stage of the 8B shape.
        {"name": "fork_samples_8b", "op": "fork", "layers": 8, "heads": 8, "head_dim": 128, "block_size": 16, "elem_bytes": 2,
         "seqs": 64, "children": 7, "length": 500},
        # A few finished sequences leave a small fp8 pool, which is then compacted.
        {"name": "retire_small", "op": "retire", "layers": 4, "heads": 1, "head_dim": 128, "block_size": 32, "elem_bytes": 1,
         "seqs": 37, "length": 90, "finished": 0.3, "spare": 0.25},
        # Half of a full batch is done; one stage of the 8B shape is compacted before a switch to fewer blocks.
        {"name": "retire_half_8b", "op": "retire", "layers": 8, "heads": 8, "head_dim": 128, "block_size": 16, "elem_bytes": 2,
         "seqs": 128, "length": 450, "finished": 0.5, "spare": 0.1},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "prompt", "fork", "retire"))
    kv_heads, group, head_dim = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 4, 5, 7, 8, 16)), rng.choice((64, 128, 128, 256))
    if kv_heads == 32:
        group = rng.choice((1, 2))
    heads = {"q_heads": kv_heads * group, "kv_heads": kv_heads, "head_dim": head_dim, "block_size": rng.choice((16, 16, 32, 64)),
             "dtype": rng.choice(("bf16", "bf16", "f16"))}
    if op == "append":
        most = max(1, min(40000, 600_000_000 // ((heads["q_heads"] + 2 * kv_heads) * head_dim)) // 2)
        total = _log(rng, 1, most)
        seqs = _log(rng, 1, min(total, 512))
        rotary = rng.choice((head_dim, head_dim, head_dim // 2, 32))
        return {"op": "append", **heads, "seqs": seqs, "new": max(1, total // seqs), "past": rng.choice((0, _log(rng, 1, 5000))),
                "ragged": rng.random() < 0.8, "norm": rng.random() < 0.5, "rotary": rotary, "interleaved": rng.random() < 0.3}
    if op == "attend":
        most = 400_000_000 // (2 * kv_heads * head_dim)
        total = min(_log(rng, 16, 400_000), most)
        seqs = _log(rng, 1, min(total, 1024))
        length = max(1, min(total // seqs, 65536))
        return {"op": "attend", **heads, "seqs": seqs, "queries": rng.choice((1, 1, 1, 1, 2, 3, 5)), "length": length,
                "spread": rng.choice(("uniform", "lognormal" if seqs <= 64 else "uniform", "fixed")) if length * seqs < 60_000 else "fixed",
                "window": rng.choice((0, 0, 0, _log(rng, 16, 2048))), "lse": rng.random() < 0.5}
    if op == "prompt":
        seqs, queries = rng.choice((1, 1, 2, 3)), _log(rng, 17, 1500)
        heads["q_heads"] = kv_heads * min(group, max(1, 32 // kv_heads))
        past = rng.choice((0, _log(rng, 1, 5000)))
        queries = min(queries, 400_000_000_000 // (4 * head_dim * heads["q_heads"] * seqs * (queries + past)))
        return {"op": "attend", **heads, "seqs": seqs, "queries": queries, "length": queries + past, "spread": "fixed",
                "window": rng.choice((0, 0, 0, _log(rng, 64, 2048))), "lse": False}
    pages = {"layers": _log(rng, 1, 8), "heads": rng.choice((1, 2, 4, 8)), "head_dim": rng.choice((64, 72, 128)), "block_size": rng.choice((16, 32)),
             "elem_bytes": rng.choice((1, 2))}
    if op == "fork":
        return {"op": "fork", **pages, "seqs": _log(rng, 1, 60), "children": rng.randint(1, 6), "length": _log(rng, 5, 450)}
    return {"op": "retire", **pages, "seqs": _log(rng, 2, 120), "length": _log(rng, 5, 400), "finished": round(rng.uniform(0.1, 0.9), 2),
            "spare": round(rng.uniform(0.0, 0.5), 2)}


# ---------------------------------------------------------------------------------------------------------------
# lengths (host arithmetic from the case and the seed alone: the largest values are the case's, the order is the seed's)
# ---------------------------------------------------------------------------------------------------------------

def _lengths(case, g):
    """Cached tokens of each sequence, new ones included."""
    n = case["seqs"]
    if case["op"] == "append":
        past = torch.full((n,), case["past"])
        new = torch.full((n,), case["new"])
        if case["ragged"]:
            past = _spread(n, case["past"] * 2, g, 0)
            new = torch.clamp(_spread(n, case["new"] * 2 - 1, g, 1), min=1) if case["new"] > 1 else new
        return past + new, new
    queries = case.get("queries", 1)
    spread = case.get("spread", "uniform")
    if spread == "fixed":
        length = torch.full((n,), case["length"])
    elif spread == "uniform":
        length = _spread(n, 2 * case["length"], g, 1)
    else:  # a fixed set of lognormal quantiles in an order of the seed's
        at = (torch.arange(n, dtype=torch.float64) + 0.5) / n
        z = torch.exp(math.sqrt(2.0) * torch.erfinv(2 * at - 1))
        length = (z / z.mean() * case["length"]).long()[torch.randperm(n, generator=g)]
    return torch.clamp(length, min=queries), torch.full((n,), queries)


def _spread(n, most, g, least):
    """n whole numbers spread evenly over [least, most], in an order of the seed's."""
    if most <= least:
        return torch.full((n,), least)
    return (least + (torch.arange(n, dtype=torch.float64) + 0.5) / n * (most - least)).long()[torch.randperm(n, generator=g)]


def _tables(lens, block_size, spare, g, rows=None):
    """A permutation of a pool's blocks dealt to the sequences: (tables [rows][widest], blocks of the pool)."""
    need = (lens + block_size - 1) // block_size
    total, widest = int(need.sum()), max(1, int(need.max()))
    pool = total + spare
    ids = torch.randperm(pool, generator=g)[:total]
    tables = torch.full((rows or len(lens), widest), -1, dtype=torch.int64)
    live = torch.arange(widest)[None, :] < need[:, None]
    tables[: len(lens)][live] = ids
    return tables.int(), pool


# ---------------------------------------------------------------------------------------------------------------
# the 4-bit format
# ---------------------------------------------------------------------------------------------------------------

def _token_bytes(d):
    return d // 2 + 4 * (d // GROUP)


def _order(d, device):
    """The dim that each place of a token's row of codes holds, for K and for V: the order in which a warp's matrix
    instructions take them."""
    n = torch.arange(d, device=device)
    t, w, i = n // (d // 4), n % (d // 4) // 8, n % 8
    k = 32 * w + 8 * (i % 4) + 2 * t + i // 4
    v = 8 * (n % (d // 8)) + n // (d // 8)
    return k, v


def _quantised(x):
    """(codes [..., D] of 0 to 15, scale and minimum [..., D/64][2] in bfloat16) of rows in 32 bits."""
    g = x.unflatten(-1, (-1, GROUP))
    u = g.amin(-1).view(torch.int32)  # the largest bfloat16 that is not above the minimum
    m = torch.where((u < 0) & (u & 0xFFFF != 0), u + 0x10000, u).bitwise_and(-0x10000).view(torch.float32).bfloat16()
    u = ((g.amax(-1) - m.float()) / 15).clamp(0, 65280).view(torch.int32)  # and the smallest that is not below the step
    s = (u + 0xFFFF).bitwise_and(-0x10000).view(torch.float32).bfloat16()
    c = torch.where(s[..., None] > 0, torch.round((g - m.float()[..., None]) / s.float()[..., None]), torch.zeros_like(g))
    return c.clamp(0, 15).to(torch.uint8).flatten(-2), torch.stack((s, m), -1)


def _packed(c, order):
    c = c[..., order]
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _values(codes, params, order):
    """Values in 32 bits of packed rows of codes [..., D/2] and their parameters [..., D/64][2]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    c = c[..., torch.argsort(order)].float().unflatten(-1, (-1, GROUP))
    p = params.float()
    return (c * p[..., 0, None] + p[..., 1, None]).flatten(-2)


def _views(pool, s):
    """The codes [K,V][block][head][tile][token][D/2] and the parameters [...][token][D/64][2] inside a pool's bytes."""
    d, h, bs = s["head_dim"], s["kv_heads"], s["block_size"]
    tiles = pool.view(2, -1, h, bs // TILE, TILE * _token_bytes(d))
    codes = tiles[..., : TILE * d // 2].unflatten(-1, (TILE, d // 2))
    params = tiles.view(torch.bfloat16)[..., TILE * d // 4:].unflatten(-1, (TILE, d // GROUP, 2))
    return codes, params


def _filled(s, blocks, g):
    """A pool of quantised K and V; channels of K differ in spread and centre, as they do after projections."""
    d, h, bs = s["head_dim"], s["kv_heads"], s["block_size"]
    pool = torch.empty(2 * blocks * h * bs * _token_bytes(d), dtype=torch.uint8, device="cuda")
    codes, params = _views(pool, s)
    spread = torch.rand(h, 1, 1, d, generator=g, device="cuda") * 1.5 + 0.3
    centre = torch.randn(h, 1, 1, d, generator=g, device="cuda") * 0.5
    piece = max(1, (1 << 27) // (h * bs * d))
    for b in range(0, blocks, piece):
        n = min(piece, blocks - b)
        for kv, order in enumerate(_order(d, "cuda")):
            x = torch.randn(n, h, bs // TILE, TILE, d, generator=g, device="cuda")
            c, p = _quantised(x * spread + centre if kv == 0 else x)
            codes[kv, b:b + n], params[kv, b:b + n] = _packed(c, order), p
    return pool


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    s = dict(case)
    host, dev = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    {"append": _prepare_append, "attend": _prepare_attend, "fork": _prepare_fork, "retire": _prepare_retire}[case["op"]](s, host, dev)
    return s


def _batch(s, lens, new, host, spare):
    tables, s["blocks"] = _tables(lens, s["block_size"], spare, host)
    s["seq_lens"], s["tables"] = lens.int().cuda(), tables.cuda()
    s["query_start"] = torch.cat((torch.zeros(1, dtype=torch.long), new.cumsum(0))).int().cuda()
    s["tokens"], s["most_queries"] = int(new.sum()), int(new.max())
    s["lens_host"], s["new_host"] = lens, new


def _prepare_append(s, host, dev):
    lens, new = _lengths(s, host)
    _batch(s, lens, new, host, 7)
    t, d, hq, hk, kind = s["tokens"], s["head_dim"], s["q_heads"], s["kv_heads"], DTYPES[s["dtype"]]
    # one projection gives q, k and v of a token side by side; a few channels are much larger than the rest
    loud = 1 + 4 * (torch.rand(hq + 2 * hk, d, generator=dev, device="cuda") < 0.03)
    s["qkv"] = (torch.randn(t, hq + 2 * hk, d, generator=dev, device="cuda") * loud).to(kind)
    s["q"], s["k"], s["v"] = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hk], s["qkv"][:, hq + hk:]
    s["q_norm"] = s["k_norm"] = None
    if s["norm"]:
        s["q_norm"], s["k_norm"] = (torch.rand(d, generator=dev, device="cuda") + 0.5 for _ in range(2))
    at = torch.arange(int(lens.max()), dtype=torch.float64, device="cuda")
    angle = at[:, None] * 500000.0 ** (-torch.arange(0, s["rotary"], 2, dtype=torch.float64, device="cuda") / s["rotary"])
    s["rope"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    s["pool"] = torch.zeros(2 * s["blocks"] * hk * s["block_size"] * _token_bytes(d), dtype=torch.uint8, device="cuda")
    s["q_out"], s["k_out"], s["v_out"] = (torch.empty(t, h, d, dtype=kind, device="cuda") for h in (hq, hk, hk))
    if own:
        import paper_2606_18741_b200 as remp
        s["cache"] = remp.make_kvq_pool(s["pool"], s["blocks"], hk, d, s["block_size"])
        s["batch"] = remp.make_kvq_batch(s["seq_lens"], s["tables"], s["query_start"], t, s["most_queries"])


def _prepare_attend(s, host, dev):
    lens, new = _lengths(s, host)
    _batch(s, lens, new, host, 5)
    t, d, kind = s["tokens"], s["head_dim"], DTYPES[s["dtype"]]
    s["pool"] = _filled(s, s["blocks"], dev)
    s["q"] = torch.randn(t, s["q_heads"], d, generator=dev, device="cuda").to(kind)
    s["scale"] = d ** -0.5
    s["out"] = torch.empty_like(s["q"])
    s["norms"] = torch.empty(t, s["q_heads"], dtype=torch.float32, device="cuda") if s["lse"] else None
    if own:
        import paper_2606_18741_b200 as remp
        s["cache"] = remp.make_kvq_pool(s["pool"], s["blocks"], s["kv_heads"], d, s["block_size"])
        s["batch"] = remp.make_kvq_batch(s["seq_lens"], s["tables"], s["query_start"], t, s["most_queries"])
        s["workspace"] = remp.make_kvq_workspace()


def _prepare_pages(s, blocks, dev):
    words = s["block_size"] * s["head_dim"] * s["elem_bytes"] // 4
    s["pool"] = torch.randint(-2 ** 31, 2 ** 31, (s["layers"], 2, blocks, s["heads"] * words), generator=dev, device="cuda", dtype=torch.int32)
    s["blocks"] = blocks
    if own:
        import paper_2606_18741_b200 as remp
        from paper_2606_18741_b200.synth import Shape, Topo
        s["topo"] = Topo(1, 1)
        s["shape"] = Shape(s["layers"], s["heads"], s["head_dim"], s["block_size"], s["elem_bytes"])
        s["shards"] = remp.make_shards([s["pool"]], [blocks])


def _refs(tables, lens, block_size, blocks):
    need = (lens + block_size - 1) // block_size
    live = torch.arange(tables.shape[1])[None, :] < need[:, None]
    return torch.bincount(tables[live].long(), minlength=blocks).int()


def _prepare_fork(s, host, dev):
    n, kids = s["seqs"], s["seqs"] * s["children"]
    lens = _spread(n, 2 * s["length"], host, 1)
    tables, blocks = _tables(lens, s["block_size"], kids + 3, host, rows=n + kids)
    every = torch.cat((lens, torch.zeros(kids, dtype=torch.long)))
    s["seq_lens"], s["tables"] = every.int().cuda(), tables.cuda()
    s["refs"] = _refs(tables, every, s["block_size"], blocks).cuda()
    s["parents"] = torch.arange(n).repeat_interleave(s["children"]).int().cuda()
    s["kids"] = (n + torch.randperm(kids, generator=host)).int().cuda()
    _prepare_pages(s, blocks, dev)
    s["refs_out"] = torch.empty_like(s["refs"])
    s["pairs"] = torch.empty(kids, 2, dtype=torch.int32, device="cuda")
    s["result"] = torch.empty(2, dtype=torch.int32, device="cuda")


def _prepare_retire(s, host, dev):
    n = s["seqs"]
    lens = _spread(n, 2 * s["length"], host, 1)
    need = int(((lens + s["block_size"] - 1) // s["block_size"]).sum())
    tables, blocks = _tables(lens, s["block_size"], 1 + int(need * s["spare"]), host)
    # every fourth sequence shares the first blocks of its neighbour, as prompts with a common start do
    for a in range(0, n - 1, 4):
        both = int(min(lens[a], lens[a + 1])) // s["block_size"] // 2
        tables[a + 1, :both] = tables[a, :both]
    s["seq_lens"], s["tables"] = lens.int().cuda(), tables.cuda()
    s["refs"] = _refs(tables, lens, s["block_size"], blocks).cuda()
    done = torch.zeros(n, dtype=torch.int32)
    done[torch.randperm(n, generator=host)[: max(1, int(n * s["finished"]))]] = 1
    s["finished"] = done.cuda()
    _prepare_pages(s, blocks, dev)
    s["lens_out"], s["tables_out"], s["refs_out"] = (torch.empty_like(s[k]) for k in ("seq_lens", "tables", "refs"))
    s["pairs"] = torch.empty((blocks + 1) // 2, 2, dtype=torch.int32, device="cuda")
    s["freed"], s["result"] = (torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(2))


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return {"append": _own_append, "attend": _own_attend, "fork": _own_fork, "retire": _own_retire}[s["op"]](s)
    return {"append": _plain_append, "attend": _plain_attend, "fork": _plain_fork, "retire": _plain_retire}[s["op"]](s)


def _own_append(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kvq_append(s["cache"], s["batch"], s["q"], s["k"], s["v"], s["q_out"], q_norm=s["q_norm"], k_norm=s["k_norm"],
                         eps=1e-6, rope=s["rope"], interleaved=s["interleaved"])
    remp.remp_kvq_read(s["cache"], s["batch"], s["k_out"], s["v_out"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kvq_attend(s["cache"], s["batch"], s["q"], s["out"], s["scale"], s["workspace"], window=s["window"], lse=s["norms"])
    return {"out": s["out"], "lse": s["norms"]} if s["lse"] else {"out": s["out"]}


def _own_fork(s):
    import paper_2606_18741_b200 as remp
    remp.remp_pages_fork(s["seq_lens"], s["tables"], s["block_size"], s["parents"], s["kids"], s["refs"], s["refs_out"], s["pairs"], s["result"])
    remp.remp_pages_copy(s["topo"], s["shape"], s["shards"], s["pairs"], s["result"])
    return {"lens": s["seq_lens"], "tables": s["tables"], "refs": s["refs_out"], "pairs": s["pairs"], "result": s["result"], "pool": s["pool"]}


def _own_retire(s):
    import paper_2606_18741_b200 as remp
    remp.remp_pages_free(s["seq_lens"], s["tables"], s["block_size"], s["finished"], s["refs"], s["lens_out"], s["tables_out"], s["refs_out"], s["freed"])
    remp.remp_pages_compact(s["lens_out"], s["tables_out"], s["block_size"], s["refs_out"], s["tables_out"], s["refs_out"], s["pairs"], s["result"])
    remp.remp_pages_copy(s["topo"], s["shape"], s["shards"], s["pairs"], s["result"])
    return {"lens": s["lens_out"], "tables": s["tables_out"], "refs": s["refs_out"], "pairs": s["pairs"], "freed": s["freed"], "result": s["result"],
            "pool": s["pool"]}


def _whose(s):
    """(sequence, position in it) of each new token."""
    t = torch.arange(s["tokens"], device="cuda")
    start = s["query_start"].long()
    seq = torch.searchsorted(start, t, right=True) - 1
    return seq, s["seq_lens"].long()[seq] - start[seq + 1] + t


def _sum_of_pairs(x):
    """The sum over the last axis, neighbours first: one order on every machine, so that a value on the edge between two
    codes falls to the same side."""
    while x.shape[-1] > 1:
        x = x[..., 0::2] + x[..., 1::2]
    return x


def _normed(x, w):
    x = x.float()
    if w is None:
        return x
    return x * (1.0 / torch.sqrt(_sum_of_pairs(x * x) / x.shape[-1] + 1e-6)) * w


def _rotated(x, cos, sin, interleaved):
    r = cos.shape[-1]
    cos, sin, a = cos[:, None], sin[:, None], x[..., : 2 * r]
    a, b = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :r], a[..., r:])
    p, q = a * cos - b * sin, b * cos + a * sin
    both = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((both, x[..., 2 * r:]), -1)


def _plain_append(s):
    seq, at = _whose(s)
    r, kind = s["rotary"] // 2, DTYPES[s["dtype"]]
    cos, sin = s["rope"][at, :r], s["rope"][at, r:]
    q = _rotated(_normed(s["q"], s["q_norm"]), cos, sin, s["interleaved"]).to(kind)
    k = _rotated(_normed(s["k"], s["k_norm"]), cos, sin, s["interleaved"])
    block = s["tables"][seq, at // s["block_size"]].long()
    tile, row = at % s["block_size"] // TILE, at % TILE
    codes, params = _views(s["pool"], s)
    ko, vo = _order(s["head_dim"], "cuda")
    (kc, kp), (vc, vp) = _quantised(k), _quantised(s["v"].float())
    codes[0, block, :, tile, row], params[0, block, :, tile, row] = _packed(kc, ko), kp
    codes[1, block, :, tile, row], params[1, block, :, tile, row] = _packed(vc, vo), vp
    return {"q": q, "k": _values(codes[0, block, :, tile, row], params[0, block, :, tile, row], ko).to(kind),
            "v": _values(codes[1, block, :, tile, row], params[1, block, :, tile, row], vo).to(kind)}


def _plain_attend(s):
    n, d, hq, hk, bs = s["seqs"], s["head_dim"], s["q_heads"], s["kv_heads"], s["block_size"]
    codes, params = _views(s["pool"], s)
    ids = s["tables"].long().clamp(min=0)
    k, v = (_values(codes[i, ids], params[i, ids], o).movedim(2, 1).reshape(n, hk, -1, d) for i, o in enumerate(_order(d, "cuda")))
    seq, at = _whose(s)
    most = s["most_queries"]
    place = torch.arange(s["tokens"], device="cuda") - s["query_start"].long()[seq]
    q = torch.zeros(n, most, hq, d, device="cuda")
    q[seq, place] = s["q"].float()
    limit = torch.full((n, most), -1, device="cuda", dtype=torch.long)
    limit[seq, place] = at
    q = q.view(n, most, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, d)
    x = q @ k.transpose(-1, -2) * s["scale"]
    key = torch.arange(k.shape[2], device="cuda")
    seen = key <= limit[..., None]
    if s["window"]:
        seen &= key > limit[..., None] - s["window"]
    x.view(n, hk, -1, most, k.shape[2]).masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x @ v) / total.clamp(min=1e-37)
    out = out.view(n, hk, -1, most, d).permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)
    out = out[seq, place].to(DTYPES[s["dtype"]])
    if not s["lse"]:
        return {"out": out}
    return {"out": out, "lse": (top + total.log()).view(n, hq, most).transpose(1, 2)[seq, place].contiguous()}


def _plain_fork(s):
    bs, parents, kids = s["block_size"], s["parents"].long(), s["kids"].long()
    lens, tables = s["seq_lens"], s["tables"]
    length = lens[parents].long()
    need = (length + bs - 1) // bs
    row = torch.where(torch.arange(tables.shape[1], device="cuda") < need[:, None], tables[parents], -1)
    part = length % bs != 0
    last = (need - 1).clamp(min=0)[:, None]
    free = torch.argsort((s["refs"] != 0).int(), stable=True)
    nth = part.cumsum(0) - 1
    source = row.gather(1, last)[:, 0]
    fresh = torch.where(part, free[nth.clamp(min=0)].int(), source)
    row.scatter_(1, last, fresh[:, None])
    lens[kids], tables[kids] = length.int(), row
    refs = s["refs"] + torch.bincount(row[row >= 0].long(), minlength=s["blocks"]).int()
    pairs = torch.full((len(kids) + 1, 2), -1, dtype=torch.int32, device="cuda")
    pairs[torch.where(part, nth, len(kids))] = torch.stack((source, fresh), 1)
    pairs[-1] = -1
    s["pool"][:, :, fresh.long()] = s["pool"][:, :, source.long()]
    return {"lens": lens, "tables": tables, "refs": refs, "pairs": pairs[:-1].contiguous(), "result": torch.stack((part.sum(), torch.zeros_like(nth[0]))).int(),
            "pool": s["pool"]}


def _plain_retire(s):
    bs, blocks, done = s["block_size"], s["blocks"], s["finished"] != 0
    live = torch.arange(s["tables"].shape[1], device="cuda") < ((s["seq_lens"] + bs - 1) // bs)[:, None]
    gone = torch.bincount(s["tables"][live & done[:, None]].long(), minlength=blocks).int()
    refs = s["refs"] - gone
    freed = ((gone > 0) & (refs == 0)).sum()
    lens = torch.where(done, 0, s["seq_lens"])
    tables = torch.where(done[:, None], -1, s["tables"])
    used = refs > 0
    count = used.sum()
    ids = torch.arange(blocks, device="cuda")
    source, target = ids[used & (ids >= count)], ids[~used & (ids < count)]
    to = ids.clone()
    to[source] = target
    tables = torch.where(live & ~done[:, None], to[tables.long().clamp(min=0)].int(), tables)
    after = torch.where(ids < count, refs, 0)
    after[target] = refs[source]
    pairs = torch.full_like(s["pairs"], -1)
    pairs[: len(source)] = torch.stack((source, target), 1).int()
    s["pool"][:, :, target] = s["pool"][:, :, source]
    zero = torch.zeros_like(count)
    return {"lens": lens, "tables": tables, "refs": after, "pairs": pairs, "freed": torch.stack((freed, zero)).int(),
            "result": torch.stack((torch.full_like(count, len(source)), zero)).int(), "pool": s["pool"]}


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    g = torch.Generator().manual_seed(1)
    if case["op"] in ("append", "attend"):
        lens, new = _lengths(case, g)
        t, d, hq, hk = int(new.sum()), case["head_dim"], case["q_heads"], case["kv_heads"]
        token = 2 * hk * _token_bytes(d)
        if case["op"] == "append":  # q, k, v in; q out; codes out; values out
            return {"bytes": t * d * 2 * (2 * hq + 4 * hk) + t * token, "flops": t * d * (hq + 2 * hk) * 10}
        # keys that some query sees, and all pairs of a query and a key that it sees
        queries, window = case["queries"], case["window"] or 1 << 60
        last = lens.tolist()
        seen = [min(n, window + queries - 1) for n in last]
        pairs = sum(min(n - i, window) for n in last for i in range(queries)) if queries < 64 else \
            sum(queries * min(n - queries / 2, window) for n in last)
        return {"bytes": sum(seen) * token + t * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}
    page = case["layers"] * 2 * case["heads"] * case["block_size"] * case["head_dim"] * case["elem_bytes"]
    lens = _spread(case["seqs"], 2 * case["length"], g, 1)
    need = (lens + case["block_size"] - 1) // case["block_size"]
    if case["op"] == "fork":
        pages = int((lens % case["block_size"] != 0).sum()) * case["children"]
        return {"bytes": 2 * pages * page + 4 * int(need.sum()) * case["children"] + 8 * int(need.sum()), "flops": 0}
    # blocks that stay, and the part of them that lies above their number (as the permutation spreads them)
    total = int(need.sum())
    pool, stay = total * (1 + case["spare"]) + 1, total * (1 - case["finished"])
    return {"bytes": 2 * page * stay * (1 - stay / pool) + 8 * total + 8 * pool, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "append":
        return _exact_append(prepare(case, seed))
    if case["op"] == "attend":
        return _exact_attend(prepare(case, seed))
    return None  # whole numbers


def _exact_rows(x, weight, cos, sin, interleaved):
    """One sequence's rows [T][H][D] in 64 bits: norm, then pairs of dims turned as complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * weight.double()
    r = cos.shape[-1]
    turn = torch.complex(cos, sin)[:, None]
    head, tail = x[..., : 2 * r], x[..., 2 * r:]
    z = torch.view_as_complex(head.unflatten(-1, (r, 2)).contiguous()) if interleaved else torch.complex(head[..., :r], head[..., r:])
    z = z * turn
    head = torch.view_as_real(z).flatten(-2) if interleaved else torch.cat((z.real, z.imag), -1)
    return torch.cat((head, tail), -1)


def _exact_held(x):
    """What 4 bits make of rows in 64 bits."""
    parts = []
    for j in range(0, x.shape[-1], GROUP):
        y = x[..., j:j + GROUP]
        least = y.min(-1, keepdim=True).values
        low = least.bfloat16()
        low = torch.where(low.double() > least, torch.nextafter(low, torch.full_like(low, -math.inf)), low).double()
        most = ((y.max(-1, keepdim=True).values - low) / 15).clamp(0, 65280)
        step = most.bfloat16()
        step = torch.where(step.double() < most, torch.nextafter(step, torch.full_like(step, math.inf)), step).double()
        code = ((y - low) / step.clamp(min=1e-300)).round().clamp(0, 15)
        parts.append(code * step + low)
    return torch.cat(parts, -1)


def _exact_append(s):
    q, k, v = [], [], []
    r, at = s["rotary"] // 2, 0
    for length, new in zip(s["lens_host"].tolist(), s["new_host"].tolist()):
        rope = s["rope"][length - new:length].double()
        mine = slice(at, at + new)
        at += new
        turn = (rope[:, :r], rope[:, r:], s["interleaved"])
        q.append(_exact_rows(s["q"][mine], s["q_norm"], *turn))
        k.append(_exact_held(_exact_rows(s["k"][mine], s["k_norm"], *turn)))
        v.append(_exact_held(s["v"][mine].double()))
    return {"q": torch.cat(q), "k": torch.cat(k), "v": torch.cat(v)}


def _exact_cached(s, kv, row, length, head):
    """K (kv 0) or V (1) of one sequence and head in 64 bits, place by place from the pool's bytes."""
    d, bs = s["head_dim"], s["block_size"]
    slices = s["pool"].view(2, s["blocks"], s["kv_heads"], -1)[kv, s["tables"][row, : (length + bs - 1) // bs].long(), head]
    tiles = slices.reshape(-1, TILE * _token_bytes(d))[: (length + TILE - 1) // TILE]
    codes = tiles[:, : TILE * d // 2].reshape(-1, d // 2)[:length].long()
    params = tiles[:, TILE * d // 2:].reshape(-1, d // GROUP, 4)[:length].long()
    scale, low = (((params[..., i] | params[..., i + 1] << 8) << 16).int().view(torch.float32).double() for i in (0, 2))
    dim = torch.arange(d, device="cuda")
    if kv == 0:
        place = dim % 8 // 2 * (d // 4) + dim // 32 * 8 + dim % 32 // 8 + dim % 2 * 4
    else:
        place = dim % 8 * (d // 8) + dim // 8
    code = codes[:, place // 2] >> (place % 2 * 4) & 15
    return code * scale[:, dim // GROUP] + low[:, dim // GROUP]


def _exact_attend(s):
    group, out, lse, at = s["q_heads"] // s["kv_heads"], [], [], 0
    if s["seqs"] * s["kv_heads"] > 20000:
        return None
    for row, (length, new) in enumerate(zip(s["lens_host"].tolist(), s["new_host"].tolist())):
        q = s["q"][at:at + new].double()
        at += new
        where = torch.arange(length - new, length, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None]
        hidden = (key > where) | (key <= where - (s["window"] or 1 << 60))
        heads, norms = [], []
        for h in range(s["kv_heads"]):
            k, v = (_exact_cached(s, i, row, length, h) for i in (0, 1))
            x = (q[:, h * group:(h + 1) * group] @ k.T * s["scale"]).masked_fill(hidden[:, None], -math.inf)
            norms.append(torch.logsumexp(x, -1))
            heads.append(torch.softmax(x, -1) @ v)
        out.append(torch.cat(heads, 1))
        lse.append(torch.cat(norms, 1))
    return {"out": torch.cat(out), "lse": torch.cat(lse)} if s["lse"] else {"out": torch.cat(out)}
