"""Plain statements in 64 bits of serving from a cache of 16-bit values and of the verification of drafts (test infrastructure)."""
from __future__ import annotations

import math

import numpy as np
import torch


class Cache:
    """A pool of 16-bit values [layers][2][blocks] with blocks [head][token][dim] or, token-major, [token][head][dim]."""

    def __init__(self, layers, blocks, heads, d, bs, dtype, token_major=False, device="cuda", gen=None):
        self.layers, self.blocks, self.heads, self.d, self.bs, self.token_major = layers, blocks, heads, d, bs, token_major
        shape = (layers, 2, blocks, bs, heads, d) if token_major else (layers, 2, blocks, heads, bs, d)
        self.data = torch.randn(shape, generator=gen, device=device).to(dtype)

    def strides(self):
        if not self.token_major:
            return None
        row = 2 * self.d
        return {"block": self.bs * self.heads * row, "head": row, "token": self.heads * row}

    def slots(self, layer, kv):
        """[block][token][head][dim], a view."""
        x = self.data[layer, kv]
        return x if self.token_major else x.transpose(1, 2)

    def rows(self, layer, kv, table, positions):
        """[position][head][dim] of one sequence in 64 bits; NaN where the block is not in the pool."""
        block = table[positions // self.bs]
        good = (block >= 0) & (block < self.blocks)
        x = self.slots(layer, kv)[block.clamp(0, self.blocks - 1).long(), positions % self.bs].double()
        x[~good] = math.nan
        return x, good


def sees(row_pos, key, window, first):
    """[rows][keys]."""
    r, k = row_pos[:, None], key[None]
    seen = k <= r
    if window > 0:
        seen = seen & ((k > r - window) | (k < first))
    return seen


def attend(cache, layer, table, length, q, first_pos, scale, window, first):
    """q [n][Hq][D] in 64 bits -> out, lse, sums of p |v| over sums of p, the most that a score's terms add up to, weights
    of every position [Hkv][length] if lse is used as it is."""
    n, hq, d = q.shape
    dev = q.device
    key = torch.arange(length, device=dev)
    k, good = cache.rows(layer, 0, table, key)
    v, _ = cache.rows(layer, 1, table, key)
    k, v = torch.where(good[:, None, None], k, 0.0), torch.where(good[:, None, None], v, 0.0)
    seen = sees(first_pos + torch.arange(n, device=dev), key, window, first) & good[None]
    hk = cache.heads
    group = hq // hk
    out, lse, size, terms = torch.zeros_like(q), torch.full((n, hq), -math.inf, dtype=torch.float64, device=dev), torch.zeros(n, hq, d, dtype=torch.float64, device=dev), 0.0
    weights = torch.zeros(hk, length, dtype=torch.float64, device=dev)
    for h in range(hq):
        kh, vh = k[:, h // group], v[:, h // group]
        hidden = ~seen.any(0)  # a slot that nobody sees may hold anything
        kh, vh = torch.where(hidden[:, None], 0.0, kh), torch.where(hidden[:, None], 0.0, vh)
        x = (q[:, h] @ kh.T * scale).masked_fill(~seen, -math.inf)
        if length:
            terms = max(terms, float((q[:, h].abs() @ kh.abs().T).max()) * scale) if n else terms
            top = x.amax(-1, keepdim=True).clamp(min=-1e300)
            p = torch.exp(x - top)
            total = p.sum(-1, keepdim=True)
            some = total[:, 0] > 0
            p = torch.where(some[:, None], p / total.clamp(min=1e-300), 0.0)
            out[:, h], size[:, h] = p @ vh, p @ vh.abs()
            lse[:, h] = torch.where(some, top[:, 0] + torch.log(total[:, 0]), -math.inf)
            weights[h // group] += p.sum(0)
    return out, lse, size, terms, weights


def choose(weights, length, keep, first, recent):
    """Positions that stay of one head: weights float32 numpy [>= length]."""
    after = min(length, keep)
    if after == length:
        return list(range(length))
    f = min(first, after)
    r = min(recent, after - f)
    inner = range(f, length - r)
    value = [(-math.inf, 1) if math.isnan(float(weights[i])) else (float(weights[i]), 0) for i in inner]
    order = sorted(range(len(inner)), key=lambda j: (value[j][1], -value[j][0], inner[j]))
    return sorted(list(range(f)) + [inner[j] for j in order[: after - f - r]] + list(range(length - r, length)))


def verify(start, drafts, target, draft, accept, pick):
    """numpy arrays in 64 bits -> tokens, accepted, word."""
    n, vocab = len(start) - 1, target.shape[1]
    tokens, accepted, word = np.full(len(drafts) + n, -1), np.zeros(n, dtype=np.int64), 0
    clean = lambda x: np.where(x > 0, x, 0.0)  # noqa: E731
    for s in range(n):
        a, b = int(start[s]), int(start[s + 1])
        k = 0
        while k < b - a:
            x = int(drafts[a + k])
            if not 0 <= x < vocab:
                word |= 2
                break
            q = clean(draft[a + k, x]) if draft is not None else 1.0
            if not accept[a + k] * q < target[a + s + k, x]:
                break
            tokens[a + s + k] = x
            k += 1
        # (the kernel looks at 32 drafts at a time and reports bad ones behind a refused one too)
        p = clean(target[a + s + k])
        w = p
        if k < b - a:
            x = int(drafts[a + k])
            if draft is not None:
                w = clean(target[a + s + k] - clean(draft[a + k]))
                w = np.where(np.isnan(w), 0.0, w)
            else:
                w = p.copy()
                if 0 <= x < vocab:
                    w[x] = 0.0
            if not w.sum() > 0:
                w = p
        sums = np.cumsum(w)
        past = np.nonzero(sums > pick[s] * sums[-1])[0]
        some = np.nonzero(w > 0)[0]
        tokens[a + s + k] = past[0] if len(past) else some[-1] if len(some) else -1
        if not len(past) and not len(some):
            word |= 4
        accepted[s] = k
    return tokens, accepted, word
