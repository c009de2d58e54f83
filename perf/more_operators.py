"""Cases for the operators that serve from a paged cache of 16-bit values between two topology switches: writing new tokens
(norm and rotation in the same pass), attention over the cache with a sliding window and first tokens that stay visible, the
weight that attention gives to every cached position, eviction by that weight, and the verification of drafted tokens.

Where `own` is false, `run` computes an operator from elementary torch operations in 32 bits (sums that pick a token in 64);
where it is true, it makes the calls of the package.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # One decode step of a full batch on the 70B shape: the new token of every sequence turned and written.
        {"name": "append_decode_70b", "op": "append", "q_heads": 64, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 256, "new": 1, "past": 120, "ragged": True, "norm": False, "rotary": 128, "interleaved": False},
        # Prompts of uneven lengths written in one go, heads of the 30B-A3B shape with its norms of queries and keys.
        {"name": "append_prompts_30b", "op": "append", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 11, "new": 2900, "past": 0, "ragged": True, "norm": True, "rotary": 128, "interleaved": False},
        # The tiny shape, lengths in [1, 256], one query each: latency.
        {"name": "attend_tiny", "op": "attend", "q_heads": 4, "kv_heads": 4, "head_dim": 64, "block_size": 16, "dtype": "f16",
         "seqs": 8, "queries": 1, "length": 128, "spread": "uniform", "window": 0, "first": 0, "lse": False},
        # A decode step over the 70B shape's long-context lognormal lengths, about 100 thousand cached tokens, with the
        # logarithms of the sums that weights and merged parts of ranks need.
        {"name": "attend_decode_70b", "op": "attend", "q_heads": 64, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 29, "queries": 1, "length": 3400, "spread": "lognormal", "window": 0, "first": 0, "lse": True},
        # Streams that have run for long: a window of their last 2048 tokens and four first ones, on the 32B shape (five query
        # heads for each KV head), three drafted tokens behind the last one.
        {"name": "attend_stream_32b", "op": "attend", "q_heads": 40, "kv_heads": 8, "head_dim": 128, "block_size": 32, "dtype": "bf16",
         "seqs": 24, "queries": 4, "length": 7001, "spread": "fixed", "window": 2048, "first": 4, "lse": False},
        # Chunks of two prompts that follow cached text, 30B-A3B heads.
        {"name": "attend_prompt_30b", "op": "attend", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 2, "queries": 2048, "length": 8191, "spread": "fixed", "window": 0, "first": 0, "lse": False},
        # The weights of one decode step added up, 8B shape.
        {"name": "weigh_decode_8b", "op": "weigh", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 37, "queries": 1, "length": 1500, "spread": "uniform", "window": 0, "first": 0},
        # The last 32 tokens of two long prompts say which of their positions matter, 30B-A3B heads.
        {"name": "weigh_prompt_30b", "op": "weigh", "q_heads": 32, "kv_heads": 4, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 2, "queries": 32, "length": 16383, "spread": "fixed", "window": 0, "first": 0},
        # A few short sequences of the tiny shape cut to 96 tokens.
        {"name": "evict_tiny", "op": "evict", "kv_heads": 4, "head_dim": 64, "block_size": 16, "dtype": "f16",
         "seqs": 5, "length": 150, "keep": 96, "first": 4, "recent": 16},
        # A batch on the 8B shape, lengths up to twice 2048, cut to 1024 tokens.
        {"name": "evict_batch_8b", "op": "evict", "kv_heads": 8, "head_dim": 128, "block_size": 16, "dtype": "bf16",
         "seqs": 41, "length": 2048, "keep": 1024, "first": 4, "recent": 128},
        # Three drafts for each of a few sequences, small vocabulary of an odd size: latency.
        {"name": "verify_small", "op": "verify", "seqs": 4, "drafts": 3, "vocab": 1999, "dtype": "f32", "given": True},
        # Up to eight drafts for each sequence of a batch, a large vocabulary.
        {"name": "verify_batch", "op": "verify", "seqs": 64, "drafts": 4, "vocab": 131072, "dtype": "f32", "given": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "prompt", "weigh", "evict", "verify"))
    if op == "verify":
        vocab = _log(rng, 200, 160_000)
        drafts = rng.choice((0, 1, 2, 3, 5))
        return {"op": "verify", "seqs": _log(rng, 3, max(3, min(200, 40_000_000 // (vocab * (2 * drafts + 1))))), "drafts": drafts, "vocab": vocab,
                "dtype": rng.choice(("f32", "f32", "bf16", "f16")), "given": rng.random() < 0.8}
    kv_heads, group, head_dim = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 4, 5, 7, 8, 16)), rng.choice((64, 128, 128, 256))
    if kv_heads == 32:
        group = rng.choice((1, 2))
    heads = {"q_heads": kv_heads * group, "kv_heads": kv_heads, "head_dim": head_dim, "block_size": rng.choice((16, 16, 32, 64)),
             "dtype": rng.choice(("bf16", "bf16", "f16"))}
    window, first = rng.choice((0, 0, _log(rng, 16, 2500))), rng.choice((0, 4, _log(rng, 1, 100)))
    if op == "append":
        most = max(1, min(40000, 600_000_000 // ((heads["q_heads"] + 2 * kv_heads) * head_dim)) // 2)
        total = _log(rng, 1, most)
        seqs = _log(rng, 1, min(total, 300))
        rotary = rng.choice((head_dim, head_dim, head_dim // 2, 32))
        return {"op": "append", **heads, "seqs": seqs, "new": max(1, total // seqs), "past": rng.choice((0, _log(rng, 1, 300))),
                "ragged": rng.random() < 0.8, "norm": rng.random() < 0.5, "rotary": rotary, "interleaved": rng.random() < 0.3}
    if op == "attend":
        total = min(_log(rng, 16, 400_000), 200_000_000 // (2 * kv_heads * head_dim))
        seqs = _log(rng, 1, min(total, 1024))
        length = max(1, min(total // seqs, 65536))
        return {"op": "attend", **heads, "seqs": seqs, "queries": rng.choice((1, 1, 1, 1, 2, 3, 5)), "length": length,
                "spread": rng.choice(("uniform", "lognormal" if seqs <= 64 else "uniform", "fixed")) if length * seqs < 60_000 else "fixed",
                "window": window, "first": first, "lse": rng.random() < 0.5}
    if op == "prompt":
        seqs, queries = rng.choice((1, 1, 2, 3)), _log(rng, 17, 1500)
        heads["q_heads"] = kv_heads * min(group, max(1, 32 // kv_heads))
        past = rng.choice((0, _log(rng, 1, 5000)))
        queries = min(queries, 300_000_000_000 // (4 * head_dim * heads["q_heads"] * seqs * (queries + past)))
        return {"op": "attend", **heads, "seqs": seqs, "queries": max(17, queries), "length": max(17, queries) + past, "spread": "fixed",
                "window": window, "first": first, "lse": False}
    if op == "weigh":
        total = min(_log(rng, 16, 100_000), 100_000_000 // (2 * kv_heads * head_dim))
        seqs = _log(rng, 1, min(total, 256))
        length = max(2, min(total // seqs, 32768))
        return {"op": "weigh", **heads, "seqs": seqs, "queries": min(length - 1, rng.choice((1, 1, 1, 3, 16, 32))) if seqs < 8 else 1, "length": length,
                "spread": rng.choice(("uniform", "fixed")) if length * seqs < 30_000 else "fixed", "window": window, "first": first}
    del heads["q_heads"]
    total = min(_log(rng, 100, 90_000), 90_000_000 // (kv_heads * head_dim))
    seqs = _log(rng, 1, max(1, min(total // 20, 200)))
    length = max(2, total // seqs // 2)
    return {"op": "evict", **heads, "seqs": seqs, "length": length, "keep": _log(rng, 2, 2 * length), "first": rng.choice((0, 1, 4)),
            "recent": rng.choice((0, 8, _log(rng, 1, length)))}


# ---------------------------------------------------------------------------------------------------------------
# lengths and tables (host arithmetic from the case and the seed alone: the largest values are the case's, the order is the
# seed's)
# ---------------------------------------------------------------------------------------------------------------

def _spread(n, most, g, least):
    """n whole numbers spread evenly over [least, most], in an order of the seed's."""
    if most <= least:
        return torch.full((n,), least)
    return (least + (torch.arange(n, dtype=torch.float64) + 0.5) / n * (most - least)).long()[torch.randperm(n, generator=g)]


def _lengths(case, g):
    """Cached tokens of each sequence, new ones included, and the new ones."""
    n = case["seqs"]
    if case["op"] == "append":
        past, new = torch.full((n,), case["past"]), torch.full((n,), case["new"])
        if case["ragged"]:
            past = _spread(n, case["past"] * 2, g, 0)
            new = torch.clamp(_spread(n, case["new"] * 2 - 1, g, 1), min=1) if case["new"] > 1 else new
        return past + new, new
    spread, queries = case.get("spread", "uniform"), case.get("queries", 1)
    if spread == "fixed":
        length = torch.full((n,), case["length"])
    elif spread == "uniform":
        length = _spread(n, 2 * case["length"], g, 1)
    else:  # a fixed set of lognormal quantiles in an order of the seed's
        at = (torch.arange(n, dtype=torch.float64) + 0.5) / n
        z = torch.exp(math.sqrt(2.0) * torch.erfinv(2 * at - 1))
        length = (z / z.mean() * case["length"]).long()[torch.randperm(n, generator=g)]
    return torch.clamp(length, min=queries), torch.full((n,), queries)


def _tables(lens, block_size, spare, g):
    """A permutation of a pool's blocks dealt to the sequences: (tables [n][widest], blocks of the pool, as many for any order
    of the lengths)."""
    need = (lens + block_size - 1) // block_size
    pool, widest = int(lens.sum()) // block_size + len(lens) + spare, max(1, int(need.max()))
    ids = torch.randperm(pool, generator=g)[: int(need.sum())]
    tables = torch.full((len(lens), widest), -1, dtype=torch.int64)
    tables[torch.arange(widest)[None, :] < need[:, None]] = ids
    return tables.int(), pool


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    s = dict(case)
    host, dev = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    {"append": _prepare_append, "attend": _prepare_attend, "weigh": _prepare_weigh, "evict": _prepare_evict,
     "verify": _prepare_verify}[case["op"]](s, host, dev)
    return s


def _batch(s, lens, new, host, spare):
    tables, s["blocks"] = _tables(lens, s["block_size"], spare, host)
    s["seq_lens"], s["tables"] = lens.int().cuda(), tables.cuda()
    s["query_start"] = torch.cat((torch.zeros(1, dtype=torch.long), new.cumsum(0))).int().cuda()
    s["tokens"], s["most_queries"] = int(new.sum()), int(new.max())
    s["lens_host"], s["new_host"] = lens, new


def _pool(s, kv, dev):
    """[K,V][block][head][token][dim]; channels of K differ in spread and centre, as they do after projections."""
    shape = (s["blocks"], s["kv_heads"], s["block_size"], s["head_dim"])
    pool = torch.empty(2, *shape, dtype=DTYPES[s["dtype"]], device="cuda")
    spread = torch.rand(s["kv_heads"], 1, s["head_dim"], generator=dev, device="cuda") * 1.5 + 0.3
    centre = torch.randn(s["kv_heads"], 1, s["head_dim"], generator=dev, device="cuda") * 0.5
    piece = max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))
    for b in range(0, s["blocks"], piece):
        for i in range(kv):
            x = torch.randn(min(piece, s["blocks"] - b), *shape[1:], generator=dev, device="cuda")
            pool[i, b:b + piece] = x * spread + centre if i == 0 else x
    return pool


def _handles(s):
    if own:
        import paper_2606_18741_b200 as remp
        s["cache"] = remp.make_kv_pool(s["pool"], s["blocks"], s["kv_heads"], s["head_dim"], s["block_size"])
        if "query_start" in s:
            s["batch"] = remp.make_kvq_batch(s["seq_lens"], s["tables"], s["query_start"], s["tokens"], s["most_queries"])
        if s["op"] == "attend":
            s["workspace"] = remp.make_kv_workspace()


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
    s["pool"] = torch.zeros(2, s["blocks"], hk, s["block_size"], d, dtype=kind, device="cuda")
    s["q_out"] = torch.empty(t, hq, d, dtype=kind, device="cuda")
    _handles(s)


def _prepare_attend(s, host, dev):
    lens, new = _lengths(s, host)
    _batch(s, lens, new, host, 5)
    s["pool"] = _pool(s, 2, dev)
    s["q"] = torch.randn(s["tokens"], s["q_heads"], s["head_dim"], generator=dev, device="cuda").to(DTYPES[s["dtype"]])
    s["scale"] = s["head_dim"] ** -0.5
    s["out"] = torch.empty_like(s["q"])
    s["norms"] = torch.empty(s["tokens"], s["q_heads"], dtype=torch.float32, device="cuda") if s["lse"] else None
    _handles(s)


def _prepare_weigh(s, host, dev):
    lens, new = _lengths(s, host)
    _batch(s, lens, new, host, 5)
    s["pool"] = _pool(s, 1, dev)
    s["q"] = torch.randn(s["tokens"], s["q_heads"], s["head_dim"], generator=dev, device="cuda").to(DTYPES[s["dtype"]])
    s["scale"] = s["head_dim"] ** -0.5
    x, _, _, seq, place = _scores(s)  # the sums that attention over the same rows has given
    most = s["most_queries"]
    norms = torch.logsumexp(x, -1).view(s["seqs"], s["q_heads"], most).transpose(1, 2)
    s["norms"] = norms[seq, place].contiguous()
    # what earlier steps have added up for each position
    s["weights"] = torch.rand(s["seqs"], s["kv_heads"], int(lens.max()), generator=dev, device="cuda") ** 8 * 5
    _handles(s)


def _prepare_evict(s, host, dev):
    lens, _ = _lengths(s, host)
    tables, s["blocks"] = _tables(lens, s["block_size"], 3, host)
    s["seq_lens"], s["tables"] = lens.int().cuda(), tables.cuda()
    s["pool"] = _pool(s, 2, dev)
    shape = (s["seqs"], s["kv_heads"], int(lens.max()))
    # a few positions have most of the weight; a tenth has none at all, so there are ties
    weights = torch.exp(2.0 * torch.randn(shape, generator=dev, device="cuda"))
    s["weights"] = torch.where(torch.rand(shape, generator=dev, device="cuda") < 0.1, 0.0, weights)
    s["weights_out"] = torch.zeros_like(s["weights"])
    s["budget"] = torch.full((s["seqs"],), s["keep"], dtype=torch.int32, device="cuda")
    s["kept"] = torch.empty(*shape[:2], min(s["keep"], shape[2]), dtype=torch.int32, device="cuda")
    s["budget"].clamp_(max=s["kept"].shape[2])
    s["longest"] = shape[2]
    _handles(s)


def _prepare_verify(s, host, dev):
    n, vocab, kind = s["seqs"], s["vocab"], DTYPES.get(s["dtype"], torch.float32)
    count = _spread(n, 2 * s["drafts"], host, 0)
    start = torch.cat((torch.zeros(1, dtype=torch.long), count.cumsum(0)))
    total = int(start[-1])
    s["draft_start"], s["total"] = start.int().cuda(), total
    # the drafting model's logits are near the target's
    logits = torch.randn(total + n, vocab, generator=dev, device="cuda") * 2.5
    s["target"] = torch.softmax(logits, -1).to(kind)
    row = torch.arange(total, device="cuda") + torch.repeat_interleave(torch.arange(n), count).cuda()
    near = logits[row] + torch.randn(total, vocab, generator=dev, device="cuda") * 0.7
    del logits
    chance = torch.softmax(near, -1)
    if total:
        # by the same draw from the sums on every machine; now and then a token that neither model favours
        at = torch.rand(total, 1, generator=dev, device="cuda", dtype=torch.float64)
        s["drafted"] = torch.searchsorted(chance.double().cumsum(-1), at).clamp(max=vocab - 1)[:, 0].int()
    else:
        s["drafted"] = torch.zeros(0, dtype=torch.int32, device="cuda")
    s["draft"] = chance.to(kind) if s["given"] else None
    s["accept"], s["pick"] = (torch.rand(k, generator=dev, device="cuda") for k in (total, n))
    s["out"] = torch.empty(total + n, dtype=torch.int32, device="cuda")
    s["accepted"] = torch.empty(n, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["op"]](s)


def _own_append(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kv_append(s["cache"], s["batch"], s["q"], s["k"], s["v"], s["q_out"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=1e-6,
                        rope=s["rope"], interleaved=s["interleaved"])
    return {"q": s["q_out"], "pool": s["pool"]}


def _own_attend(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kv_attend(s["cache"], s["batch"], s["q"], s["out"], s["scale"], s["workspace"], window=s["window"], first=s["first"],
                        lse=s["norms"])
    return {"out": s["out"], "lse": s["norms"]} if s["lse"] else {"out": s["out"]}


def _own_weigh(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kv_weigh(s["cache"], s["batch"], s["q"], s["norms"], s["weights"], s["scale"], window=s["window"], first=s["first"])
    return {"weights": s["weights"]}


def _own_evict(s):
    import paper_2606_18741_b200 as remp
    remp.remp_kv_evict(s["cache"], s["seq_lens"], s["tables"], s["budget"], s["weights"], s["weights_out"], s["kept"], first=s["first"],
                       recent=s["recent"], max_tokens=s["longest"])
    return {"kept": s["kept"], "weights": s["weights_out"], "pool": s["pool"]}


def _own_verify(s):
    import paper_2606_18741_b200 as remp
    remp.remp_draft_verify(s["draft_start"], s["drafted"], s["target"], s["draft"], s["accept"], s["pick"], s["out"], s["accepted"])
    return {"tokens": s["out"], "accepted": s["accepted"]}


_OWN = {"append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict, "verify": _own_verify}


def _whose(s):
    """(sequence, position in it) of each new token."""
    t = torch.arange(s["tokens"], device="cuda")
    start = s["query_start"].long()
    seq = torch.searchsorted(start, t, right=True) - 1
    return seq, s["seq_lens"].long()[seq] - start[seq + 1] + t


def _normed(x, w):
    x = x.float()
    return x if w is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _rotated(x, cos, sin, interleaved):
    r = cos.shape[-1]
    cos, sin, a = cos[:, None], sin[:, None], x[..., : 2 * r]
    a, b = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :r], a[..., r:])
    p, q = a * cos - b * sin, b * cos + a * sin
    both = torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)
    return torch.cat((both, x[..., 2 * r:]), -1)


def _plain_append(s):
    seq, at = _whose(s)
    r, kind, bs = s["rotary"] // 2, DTYPES[s["dtype"]], s["block_size"]
    cos, sin = s["rope"][at, :r], s["rope"][at, r:]
    block = s["tables"][seq, at // bs].long()
    s["pool"][0, block, :, at % bs] = _rotated(_normed(s["k"], s["k_norm"]), cos, sin, s["interleaved"]).to(kind)
    s["pool"][1, block, :, at % bs] = s["v"]
    return {"q": _rotated(_normed(s["q"], s["q_norm"]), cos, sin, s["interleaved"]).to(kind), "pool": s["pool"]}


def _cached(s, kv):
    """K or V of every sequence in 32 bits, [sequence][head][position][dim], padded to the longest."""
    x = s["pool"][kv, s["tables"].long().clamp(min=0)].float()
    return x.movedim(2, 1).reshape(s["seqs"], s["kv_heads"], -1, s["head_dim"])


def _scores(s):
    """Scaled scores [sequence][KV head][query head of it x row][position] (-inf: not seen), what is seen, positions, whose rows."""
    n, d, hq, hk, most = s["seqs"], s["head_dim"], s["q_heads"], s["kv_heads"], s["most_queries"]
    k = _cached(s, 0)
    seq, at = _whose(s)
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
        seen &= (key > limit[..., None] - s["window"]) | (key < s["first"])
    x.view(n, hk, -1, most, k.shape[2]).masked_fill_(~seen[:, None, None], -math.inf)
    return x, seen, limit, seq, place


def _plain_attend(s):
    n, d, hq, most = s["seqs"], s["head_dim"], s["q_heads"], s["most_queries"]
    x, _, _, seq, place = _scores(s)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x @ _cached(s, 1)) / total.clamp(min=1e-37)
    out = out.view(n, s["kv_heads"], -1, most, d).permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)
    out = out[seq, place].to(DTYPES[s["dtype"]])
    if not s["lse"]:
        return {"out": out}
    return {"out": out, "lse": (top + total.log()).view(n, hq, most).transpose(1, 2)[seq, place].contiguous()}


def _plain_weigh(s):
    n, hq, hk, most = s["seqs"], s["q_heads"], s["kv_heads"], s["most_queries"]
    x, seen, limit, seq, place = _scores(s)
    norms = torch.zeros(n, most, hq, device="cuda")
    norms[seq, place] = s["norms"]
    norms = norms.permute(0, 2, 1).reshape(n, hk, -1, 1)
    longest = s["weights"].shape[2]
    added = (x - norms).exp_().sum(2)[..., :longest]
    key = torch.arange(longest, device="cuda")
    lens = s["seq_lens"].long()[:, None]
    new = key >= lens - (s["query_start"][1:] - s["query_start"][:-1]).long()[:, None]
    before = s["weights"]
    s["weights"].copy_(torch.where((key < lens)[:, None], torch.where(new[:, None], 0.0, before) + added, before))
    return {"weights": s["weights"]}


def _plain_evict(s):
    n, hk, bs, longest, room = s["seqs"], s["kv_heads"], s["block_size"], s["longest"], s["kept"].shape[2]
    key, lens, budget = torch.arange(longest, device="cuda"), s["seq_lens"].long()[:, None], s["budget"].long()[:, None]
    after = torch.minimum(lens, budget)
    # what stays whatever its weight: the first tokens, then the last ones, as far as the budget goes
    first = after.clamp(max=s["first"])
    recent = (after - first).clamp(max=s["recent"])
    rank = torch.where((key < first) | ((key >= lens - recent) & (key < lens)), math.inf, -math.inf)
    rank = torch.where(((key >= first) & (key < lens - recent))[:, None], s["weights"], rank[:, None])
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)[..., :room]  # equal weights: the lower position first
    order = torch.where((torch.arange(room, device="cuda") < after)[:, None], order, longest).sort(-1).values
    stays = order < longest
    s["kept"].copy_(torch.where(stays, order, -1))
    order = order.clamp(max=longest - 1)
    s["weights_out"][..., :room] = torch.where(stays, s["weights"].gather(-1, order), s["weights_out"][..., :room])
    # rows that move, K and V of every head
    seq, head, to = (stays & (s["kept"] != torch.arange(room, device="cuda"))).nonzero(as_tuple=True)
    source = order[seq, head, to]
    tables = s["tables"].long()
    at, by = tables[seq, source // bs], tables[seq, to // bs]
    s["pool"][:, by, head, to % bs] = s["pool"][:, at, head, source % bs]
    return {"kept": s["kept"], "weights": s["weights_out"], "pool": s["pool"]}


def _plain_verify(s):
    n, total, vocab, start = s["seqs"], s["total"], s["vocab"], s["draft_start"].long()
    count = start[1:] - start[:-1]
    i = torch.arange(total, device="cuda")
    seq = torch.searchsorted(start, i, right=True) - 1
    drafted = s["drafted"].long()
    p = s["target"][i + seq, drafted].double()
    q = s["draft"][i, drafted].double() if s["given"] else torch.ones_like(p)
    refused = s["accept"].double() * q >= p
    # drafts before the first refusal of their sequence
    at = torch.where(refused, i - start[seq], total + 1)
    accepted = count.scatter_reduce(0, seq, at, "amin")
    row = start[:-1] + torch.arange(n, device="cuda") + accepted
    w = s["target"][row].double()
    cut = accepted < count
    if total:
        of = (start[:-1] + accepted).clamp(max=total - 1)
        less = s["draft"][of].double() if s["given"] else torch.zeros_like(w).scatter_(1, drafted[of, None], 2.0)
        rest = (w - less).clamp(min=0) * cut[:, None]
        w = torch.where(rest.sum(-1, keepdim=True) > 0, rest, w)
    sums = w.cumsum(-1)
    pick = torch.searchsorted(sums, s["pick"].double()[:, None] * sums[:, -1:], right=True).clamp(max=vocab - 1)
    out = torch.full((total + n,), -1, dtype=torch.int32, device="cuda")
    keep = i - start[seq] < accepted[seq]
    out[(i + seq)[keep]] = s["drafted"][keep]
    out[row] = pick[:, 0].int()
    return {"tokens": out, "accepted": accepted.int()}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict, "verify": _plain_verify}


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    g = torch.Generator().manual_seed(1)
    if case["op"] == "verify":  # one row of each sequence, two where a draft is refused (about half of them)
        rows = case["seqs"] * (1.5 if case["given"] and case["drafts"] else 1.0)
        return {"bytes": rows * case["vocab"] * (4 if case["dtype"] == "f32" else 2), "flops": 2 * rows * case["vocab"]}
    lens, new = _lengths(case, g)
    d, hk = case["head_dim"], case["kv_heads"]
    if case["op"] == "evict":
        cut = lens > case["keep"]
        moved = int(cut.sum()) * max(0, case["keep"] - case["first"])
        return {"bytes": moved * hk * d * 2 * 2 * 2 + 4 * hk * int(lens.sum()) + 8 * hk * int(lens.clamp(max=case["keep"]).sum()), "flops": 0}
    t, hq = int(new.sum()), case["q_heads"]
    if case["op"] == "append":  # q, k, v in; q, k, v out
        return {"bytes": t * d * 4 * (hq + 2 * hk), "flops": t * d * (hq + 2 * hk) * 8}
    # keys that some query sees, and all pairs of a query and a key that it sees
    queries, window, first = case["queries"], case["window"] or 1 << 60, case["first"]
    seen = pairs = 0
    for m in lens.tolist():
        seen += min(m, window + queries - 1 + first)
        pairs += sum(min(m - i, min(m - i, window) + first) for i in range(queries))
    if case["op"] == "weigh":
        return {"bytes": seen * hk * (2 * d + 8) + t * hq * (2 * d + 4), "flops": 2 * d * hq * pairs}
    return {"bytes": seen * hk * 4 * d + t * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "append":
        return _exact_append(prepare(case, seed))
    if case["op"] in ("attend", "weigh"):
        return None if case["seqs"] * case["kv_heads"] > 12000 else _exact_attention(prepare(case, seed))
    return None  # whole numbers and copies


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


def _exact_append(s):
    q, pool, at = [], s["pool"].double(), 0
    r, bs = s["rotary"] // 2, s["block_size"]
    for row, (length, new) in enumerate(zip(s["lens_host"].tolist(), s["new_host"].tolist())):
        rope = s["rope"][length - new:length].double()
        mine = slice(at, at + new)
        at += new
        turn = (rope[:, :r], rope[:, r:], s["interleaved"])
        q.append(_exact_rows(s["q"][mine], s["q_norm"], *turn))
        where = torch.arange(length - new, length, device="cuda")
        block = s["tables"][row, where // bs].long()
        pool[0, block, :, where % bs] = _exact_rows(s["k"][mine], s["k_norm"], *turn)
        pool[1, block, :, where % bs] = s["v"][mine].double()
    return {"q": torch.cat(q), "pool": pool}


def _exact_attention(s):
    """Attention, or the weights of every position, from the definition."""
    group, out, lse, at, bs = s["q_heads"] // s["kv_heads"], [], [], 0, s["block_size"]
    weights = s["weights"].double() if s["op"] == "weigh" else None
    for row, (length, new) in enumerate(zip(s["lens_host"].tolist(), s["new_host"].tolist())):
        q = s["q"][at:at + new].double()
        where = torch.arange(length - new, length, device="cuda")[:, None]
        key = torch.arange(length, device="cuda")[None]
        near = (where - key < s["window"]) if s["window"] else torch.ones_like(key, dtype=torch.bool)
        hidden = ~((key <= where) & (near | (key < s["first"])))
        blocks = s["tables"][row, : (length + bs - 1) // bs].long()
        heads, norms = [], []
        for h in range(s["kv_heads"]):
            k = s["pool"][0, blocks, h].reshape(-1, s["head_dim"])[:length].double()
            x = (q[:, h * group:(h + 1) * group] @ k.T * s["scale"]).masked_fill(hidden[:, None], -math.inf)
            if weights is not None:
                weights[row, h, length - new:length] = 0
                weights[row, h, :length] += torch.exp(x - s["norms"][at:at + new, h * group:(h + 1) * group, None].double()).sum((0, 1))
                continue
            norms.append(torch.logsumexp(x, -1))
            heads.append(torch.softmax(x, -1) @ s["pool"][1, blocks, h].reshape(-1, s["head_dim"])[:length].double())
        at += new
        if weights is None:
            out.append(torch.cat(heads, 1))
            lse.append(torch.cat(norms, 1))
    if weights is not None:
        return {"weights": weights}
    return {"out": torch.cat(out), "lse": torch.cat(lse)} if s["lse"] else {"out": torch.cat(out)}
