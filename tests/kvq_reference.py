"""Plain statements of the 4-bit cache, of attention over it and of page management (numpy; test infrastructure)."""
from __future__ import annotations

import numpy as np

F = np.float32


def token_bytes(d: int) -> int:
    return d // 2 + d // 16


def bf16_below(x: np.ndarray) -> np.ndarray:
    """float32 -> bits of the largest bfloat16 that is not above it."""
    u = np.ascontiguousarray(x, dtype=F).view(np.uint32).astype(np.int64)
    return ((u + np.where((u >> 31 == 1) & (u & 0xFFFF != 0), 0x10000, 0)) >> 16).astype(np.uint16)


def bf16_above(x: np.ndarray) -> np.ndarray:
    """float32 >= 0 -> bits of the smallest bfloat16 that is not below it."""
    u = np.ascontiguousarray(x, dtype=F).view(np.uint32).astype(np.int64)
    return ((u + 0xFFFF) >> 16).astype(np.uint16)


def bf16_value(bits: np.ndarray) -> np.ndarray:
    return (bits.astype(np.uint32) << 16).view(F)


def place_of(d: int, is_v: bool) -> np.ndarray:
    """place_of[n] = the dim that place n of a token's codes holds (the formulas of the header)."""
    n = np.arange(d)
    if is_v:
        return 8 * (n % (d // 8)) + n // (d // 8)
    return 32 * ((n % (d // 4)) // 8) + 8 * (n % 4) + 2 * (n // (d // 4)) + (n % 8) // 4


def quantise(x: np.ndarray):
    """float32 rows [..., D] -> codes [..., D], bfloat16 bits of steps and minima [..., D/64], one float32 operation at a time."""
    g = x.astype(F).reshape(x.shape[:-1] + (-1, 64))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], F(0), g)
    m = bf16_below(g.min(-1))
    mf = bf16_value(m)
    s = bf16_above(np.minimum(np.maximum((g.max(-1) - mf) * (F(1) / F(15)), F(0)), F(65280)))
    sf = bf16_value(s)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(sf[..., None] > 0, np.rint((g - mf[..., None]) / sf[..., None]), 0)
    c = np.clip(c, 0, 15).astype(np.uint8)
    m, s = np.where(bad, 0x7FC0, m).astype(np.uint16), np.where(bad, 0, s).astype(np.uint16)
    c[bad] = 0
    return c.reshape(x.shape), s, m


def norm_rows(x: np.ndarray, w, eps: float) -> np.ndarray:
    x = x.astype(F)
    if w is None:
        return x
    s = x * x
    while s.shape[-1] > 1:
        s = s[..., 0::2] + s[..., 1::2]
    r = F(1) / np.sqrt(s / F(x.shape[-1]) + F(eps))
    return x * r * w.astype(F)


def turn_rows(x: np.ndarray, rope, at: np.ndarray, interleaved: bool) -> np.ndarray:
    """x [T][H][D], rope [rows][rotary_dim], at [T]."""
    if rope is None:
        return x
    r = rope.shape[1] // 2
    cos, sin = rope[at, None, :r], rope[at, None, r:]
    out = x.copy()
    ia, ib = (np.arange(0, 2 * r, 2), np.arange(1, 2 * r, 2)) if interleaved else (np.arange(r), np.arange(r, 2 * r))
    a, b = x[..., ia], x[..., ib]
    out[..., ia] = a * cos - b * sin
    out[..., ib] = b * cos + a * sin
    return out


class Pool:
    """A 4-bit pool [layers][2][blocks][heads][slice] as bytes."""

    def __init__(self, layers, blocks, heads, d, bs, fill=0xA5):
        self.shape = (layers, 2, blocks, heads, bs // 16, 16 * token_bytes(d))
        self.d, self.bs, self.heads, self.blocks, self.layers = d, bs, heads, blocks, layers
        self.bytes = np.full(self.shape, fill, dtype=np.uint8)

    def write(self, layer, kv, block, pos, x):
        """x float32 [heads][D] at position pos of its sequence, in `block`."""
        d = self.d
        c, s, m = quantise(x)
        c = c[:, place_of(d, kv == 1)]
        tile, row = pos % self.bs // 16, pos % 16
        at = self.bytes[layer, kv, block, :, tile]
        at[:, row * d // 2:(row + 1) * d // 2] = c[:, 0::2] | c[:, 1::2] << 4
        par = np.stack([s, m], -1).reshape(self.heads, -1).view(np.uint8)
        o = 8 * d + row * d // 16
        at[:, o:o + d // 16] = par

    def read(self, layer, kv, block, pos):
        """float64 [heads][D]."""
        d = self.d
        tile, row = pos % self.bs // 16, pos % 16
        at = self.bytes[layer, kv, block, :, tile]
        b = at[:, row * d // 2:(row + 1) * d // 2]
        n = np.stack([b & 15, b >> 4], -1).reshape(self.heads, d)
        c = np.empty_like(n)
        c[:, place_of(d, kv == 1)] = n
        o = 8 * d + row * d // 16
        par = np.ascontiguousarray(at[:, o:o + d // 16]).view(np.uint16).reshape(self.heads, d // 64, 2)
        s, m = bf16_value(par[..., 0]).astype(np.float64), bf16_value(par[..., 1]).astype(np.float64)
        return c * np.repeat(s, 64, -1) + np.repeat(m, 64, -1)

    def rows(self, layer, kv, table, length):
        """float64 [length][heads][D] of one sequence; blocks outside the pool give NaN."""
        out = np.full((length, self.heads, self.d), np.nan)
        for p in range(length):
            b = table[p // self.bs]
            if 0 <= b < self.blocks:
                out[p] = self.read(layer, kv, b, p)
        return out


def attend(q, k, v, first_pos, scale, window):
    """q [n][Hq][D], k and v [len][Hkv][D] in 64 bits (NaN rows: not there) -> out [n][Hq][D], lse [n][Hq], and what bounds the
    rounding: sums of p * (spread of v's row), sums of p * (largest of v's row), and the most that a score moves where keys
    are rounded to 11 bits."""
    n, hq, d = q.shape
    length, hk, _ = k.shape
    out, lse, weight, size, move = np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq)), np.zeros((n, hq)), np.zeros((n, hq))
    key = np.arange(length)
    for i in range(n):
        pos = first_pos + i
        seen = (key <= pos) & ~np.isnan(k[:, 0, 0] if length else np.zeros(0))
        if window > 0:
            seen &= key > pos - window
        if not seen.any():
            continue
        for h in range(hq):
            kk, vv = k[seen, h * hk // hq], v[seen, h * hk // hq]
            x = kk @ q[i, h] * scale
            top = x.max()
            e = np.exp(x - top)
            out[i, h] = e @ vv / e.sum()
            lse[i, h] = top + np.log(e.sum())
            weight[i, h] = (e @ (vv.max(-1) - vv.min(-1))) / e.sum()
            size[i, h] = (e @ np.abs(vv).max(-1)) / e.sum()
            move[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max() * 2.0 ** -11
    return out, lse, weight, size, move


# ---- pages ----

def need_of(length, bs):
    return -(-length // bs)


def refs_of(lens, tables, bs, blocks):
    refs = np.zeros(blocks, dtype=np.int32)
    for s, n in enumerate(lens):
        for b in tables[s, :need_of(int(n), bs)]:
            if 0 <= b < blocks:
                refs[b] += 1
    return refs


def fork(lens, tables, bs, parents, children, refs):
    lens, tables, out = lens.copy(), tables.copy(), refs.copy()
    free = [i for i in range(len(refs)) if refs[i] == 0]
    pairs = np.full((len(children), 2), -1, dtype=np.int32)
    need = sum(1 for p in parents if lens[p] % bs)
    if need > len(free):
        return lens, tables, out, pairs, [0, 1]
    k = 0
    for p, c in zip(parents, children):
        n = need_of(int(lens[p]), bs)
        row = np.full(tables.shape[1], -1, dtype=np.int32)
        row[:n] = tables[p, :n]
        if lens[p] % bs:
            pairs[k] = row[n - 1], free[k]
            row[n - 1] = free[k]
            k += 1
        for b in row[:n]:
            out[b] += 1
        tables[c], lens[c] = row, lens[p]
    return lens, tables, out, pairs, [k, 0]


def free(lens, tables, bs, finished, refs):
    lens, tables, refs = lens.copy(), tables.copy(), refs.copy()
    before = refs.copy()
    for s in np.nonzero(finished)[0]:
        for b in tables[s, :need_of(int(lens[s]), bs)]:
            refs[b] -= 1
        tables[s], lens[s] = -1, 0
    return lens, tables, refs, [int(((before > 0) & (refs == 0)).sum()), 0]


def compact(lens, tables, bs, refs, max_pairs):
    blocks = len(refs)
    total = int((refs > 0).sum())
    movers = [i for i in range(total, blocks) if refs[i] > 0]
    holes = [i for i in range(total) if refs[i] <= 0]
    to = {a: b for a, b in zip(movers, holes)}
    tables, out = tables.copy(), np.zeros_like(refs)
    for s, n in enumerate(lens):
        for j in range(need_of(int(n), bs)):
            tables[s, j] = to.get(int(tables[s, j]), tables[s, j])
    out[:total] = refs[:total]
    for a, b in to.items():
        out[b] = refs[a]
    pairs = np.full((max_pairs, 2), -1, dtype=np.int32)
    for i, (a, b) in enumerate(to.items()):
        pairs[i] = a, b
    return tables, out, pairs, [len(movers), 0]
