"""CPU oracle of the paged key/value cache and the attention over it.

TEST INFRASTRUCTURE ONLY, like the other oracles: plain NumPy, no code shared with the HIP path, nothing imported from
the package.

A cache is a dict of arrays: k, v [pages, kv heads, page tokens, row] (float32, float16 or int8), for int8 also k_scale,
v_scale [pages, kv heads, page tokens], and table [states, table pages].  Slot j of state b is row j % page tokens of page
table[b, j // page tokens]; a page number outside the pool makes its slots disappear.

What is rounded: append rotates in fp32, each operation rounded once in the written order (a c - b s, b c + a s), and
rounds to the cache's type once.  Attention, weights and everything that follows from them are fp64.  Selection and
moving are exact.  The paper (Sec. 3.1, Eq. 3) has neither a cache nor eviction: the attention is that of
bitrl_oracle.causal_gqa_attention, split at the cache, and eviction keeps what got most attention.
"""
from __future__ import annotations

import numpy as np

F32 = np.float32
SMALLEST = F32(1e-30)


def place(cache, b, slot):
    """(page, row in page) of a slot, or None where there is none."""
    tokens = cache["k"].shape[2]
    if slot < 0 or slot // tokens >= cache["table"].shape[1]:
        return None
    page = int(cache["table"][b, slot // tokens])
    if not 0 <= page < cache["k"].shape[0]:
        return None
    return page, slot % tokens


def rotate(x, cos, sin):
    """x [heads, dh] fp32 by cos, sin [dh / 2] fp32, each operation rounded to fp32."""
    half = x.shape[-1] // 2
    a, b = x[..., :half].astype(F32), x[..., half:].astype(F32)
    return np.concatenate([(a * cos) - (b * sin), (b * cos) + (a * sin)], axis=-1).astype(F32)


def quantise_row(x):
    """int8 codes and fp32 scale of one row; zeros under a scale that is infinite or NaN where a component is."""
    a = np.maximum(np.abs(x).max(), SMALLEST).astype(F32)
    if not np.isfinite(a):
        return np.zeros(x.shape, dtype=np.int8), F32(a / F32(127))
    codes = np.clip(np.rint((x * (F32(127) / a)).astype(F32)), -127, 127).astype(np.int8)
    return codes, F32(a / F32(127))


def tokens_of(cu, lens, b, T):
    """(first row, new tokens, first slot) of state b; cu None: T / B each."""
    if cu is None:
        n = T // len(lens)
        return b * n, n, int(lens[b]) - n
    n = int(cu[b + 1]) - int(cu[b])
    return int(cu[b]), n, int(lens[b]) - n


def append(cache, qkv, hq, cu, lens, positions, cos, sin):
    """Writes the new tokens' rows into the cache's arrays."""
    dh = cos.shape[1] * 2
    hkv = cache["k"].shape[1]
    rows = qkv.reshape(qkv.shape[0], hq + 2 * hkv, dh)
    for b in range(len(lens)):
        r0, n, base = tokens_of(cu, lens, b, qkv.shape[0])
        for i in range(n):
            at = place(cache, b, base + i)
            if at is None:
                continue
            p = base + i if positions is None else int(positions[r0 + i])
            p = min(max(p, 0), cos.shape[0] - 1)
            k, v = rotate(rows[r0 + i, hq:hq + hkv], cos[p], sin[p]), rows[r0 + i, hq + hkv:]
            for name, x in (("k", k), ("v", v)):
                cache[name][at[0], :, at[1], dh:] = 0
                if cache[name].dtype == np.int8:
                    for h in range(hkv):
                        cache[name][at[0], h, at[1], :dh], cache[name + "_scale"][at[0], h, at[1]] = quantise_row(x[h])
                else:
                    cache[name][at[0], :, at[1], :dh] = x.astype(cache[name].dtype)


def sees(i, n, base, slot, tree_row):
    """Whether new token i sees a slot."""
    if tree_row is None:
        return slot <= base + i
    j = slot - base
    if j < 0:
        return True
    return j // 32 < len(tree_row) and bool((int(tree_row[j // 32]) >> (j % 32)) & 1)


def attend(cache, qkv, hq, cu, lens, positions, cos, sin, tree=None):
    """(out [T, hq * dh], weights added [B, kv heads, longest], reach [T]) in fp64; rows of no state are NaN.

    reach: the largest sum_j p_j |v_j| over a token's heads and components.  Relative errors of at most eps on every
    probability move an output by at most eps times that."""
    dh = cos.shape[1] * 2
    hkv, T = cache["k"].shape[1], qkv.shape[0]
    group = hq // hkv
    out = np.full((T, hq, dh), np.nan)
    longest = max(1, max(int(x) for x in lens))
    weights = np.zeros((len(lens), hkv, longest))
    reach = np.zeros(T)
    c64, s64 = cos.astype(np.float64), sin.astype(np.float64)
    rows = qkv.reshape(T, hq + 2 * hkv, dh).astype(np.float64)
    for b in range(len(lens)):
        r0, n, base = tokens_of(cu, lens, b, T)
        slots, where = [], []
        for slot in range(int(lens[b])):
            at = place(cache, b, slot)
            if at is not None:
                slots.append(slot)
                where.append(at)
        slots = np.array(slots, dtype=np.int64)
        if len(slots):
            pg, off = np.array(where).T
            k = cache["k"][pg, :, off, :dh].astype(np.float64)           # [slots, kv heads, dh]
            v = cache["v"][pg, :, off, :dh].astype(np.float64)
            if "k_scale" in cache:
                k = k * cache["k_scale"][pg, :, off].astype(np.float64)[..., None]
                v = v * cache["v_scale"][pg, :, off].astype(np.float64)[..., None]
        for i in range(n):
            p = base + i if positions is None else int(positions[r0 + i])
            p = min(max(p, 0), cos.shape[0] - 1)
            see = np.array([sees(i, n, base, int(s), None if tree is None else tree[r0 + i]) for s in slots], dtype=bool)
            for h in range(hq):
                if not see.any():
                    out[r0 + i, h] = 0
                    continue
                a, c = rows[r0 + i, h, :dh // 2], rows[r0 + i, h, dh // 2:]
                q = np.concatenate([a * c64[p] - c * s64[p], c * c64[p] + a * s64[p]])
                x = k[see][:, h // group] @ q / np.sqrt(dh)
                e = np.exp(x - x.max())
                e /= e.sum()
                out[r0 + i, h] = e @ v[see][:, h // group]
                reach[r0 + i] = max(reach[r0 + i], (e @ np.abs(v[see][:, h // group])).max())
                weights[b, h // group, slots[see]] += e
    return out.reshape(T, hq * dh), weights, reach


def select(weights, lens, keep, first, recent):
    """(kept [B, heads, keep], counts [B])."""
    B, H, _ = weights.shape
    kept = np.full((B, H, keep), -1, dtype=np.int32)
    counts = np.minimum(np.maximum(lens, 0), keep).astype(np.int32)
    for b in range(B):
        n = max(int(lens[b]), 0)
        for h in range(H):
            if n <= keep:
                kept[b, h, :n] = np.arange(n)
                continue
            w = [float("-inf") if np.isnan(x) else float(x) for x in weights[b, h, :n]]
            middle = sorted(range(first, n - recent), key=lambda j: (-w[j], j))[:keep - first - recent]
            kept[b, h] = sorted(list(range(first)) + middle + list(range(n - recent, n)))
    return kept, counts


def compact(cache, lens, kept, start, counts, weights=None):
    """Moves rows (and weights [B, heads, slots]) in the given arrays."""
    for b in range(len(lens)):
        n = max(int(lens[b]), 0)
        s0 = 0 if start is None else min(max(int(start[b]), 0), n)
        for h in range(cache["k"].shape[1]):
            lst = kept[b, h if kept.shape[1] > 1 else 0]
            for i in range(min(max(int(counts[b]), 0), len(lst), n - s0)):
                src, dst = int(lst[i]), s0 + i
                if src <= dst or src >= n:
                    continue
                if weights is not None:
                    weights[b, h, dst] = weights[b, h, src]
                x, y = place(cache, b, src), place(cache, b, dst)
                if x is None or y is None:
                    continue
                for name in ("k", "v", "k_scale", "v_scale"):
                    if name in cache:
                        cache[name][y[0], h, y[1]] = cache[name][x[0], h, x[1]]
