"""Plain numpy oracle of a worker's step: prefix groups, block tables and slot
map, cache writes, attention over the block cache in 64 bits.

TEST INFRASTRUCTURE ONLY, like the rest of this folder: loops over requests,
entries and tokens, straight from the definitions in include/rkroute.h.
"""
from __future__ import annotations

import numpy as np

BLOCK = 16


def common_blocks(a, b) -> int:
    """Leading blocks that two chains have in common; a hash of 0 is missing, and in common with none."""
    n = 0
    while n < min(len(a), len(b)) and a[n] == b[n] and a[n] != 0:
        n += 1
    return n


def prefix_groups(chains, chain_off, min_blocks):
    """(order, group_off, shared, n_groups), padded as the library pads them."""
    B = len(chain_off) - 1
    chain = [chains[chain_off[i]:chain_off[i + 1]] for i in range(B)]
    members = {}
    for i in range(B):
        named = len(chain[i]) >= min_blocks and int(chain[i][min_blocks - 1]) != 0
        members.setdefault(("hash", int(chain[i][min_blocks - 1])) if named else ("own", i), []).append(i)
    groups = sorted(members.values(), key=lambda m: m[0])
    order = [i for m in groups for i in m]
    off = np.full(B + 1, B, np.int64)
    shared = np.zeros(B, np.int32)
    at = 0
    for g, m in enumerate(groups):
        off[g] = at
        at += len(m)
        if len(m) > 1:
            shared[g] = min(common_blocks(chain[i], chain[m[0]]) for i in m)
    return np.array(order, np.int32), off, shared, len(groups)


def leads(kv_len, group_off, shared):
    """Of each request: the first of its group, and how many blocks that one lends it."""
    B = len(kv_len)
    first, lead = np.arange(B), np.zeros(B, np.int64)
    if group_off is not None:
        for g in range(B):
            for i in range(group_off[g], group_off[g + 1]):
                first[i] = group_off[g]
                if i != first[i]:
                    lead[i] = min(shared[g], kv_len[first[i]] // BLOCK)
    return first, lead


def block_tables(tables, kv_len, new_len, have, free_blocks, n_slots, group_off=None, shared=None):
    """(tables, slots, q_off, taken) after the step; no bad lengths here."""
    tables = tables.copy()
    first, lead = leads(kv_len, group_off, shared)
    slots = np.full(n_slots, -1, np.int64)
    q_off = np.zeros(len(kv_len) + 1, np.int64)
    taken = 0
    for i in range(len(kv_len)):
        for p in range(have[i], -(-int(kv_len[i]) // BLOCK)):
            if p < lead[i]:
                tables[i, p] = tables[first[i], p]
            else:
                tables[i, p] = free_blocks[taken] if taken < len(free_blocks) else -1
                taken += taken < len(free_blocks)
        q_off[i + 1] = q_off[i] + new_len[i]
        for t in range(new_len[i]):
            x = int(kv_len[i] - new_len[i] + t)
            p = x // BLOCK
            if q_off[i] + t < n_slots and not have[i] <= p < lead[i] and tables[i, p] >= 0:
                slots[q_off[i] + t] = BLOCK * int(tables[i, p]) + x % BLOCK
    return tables, slots, q_off, taken


def attention(q, k_cache, v_cache, tables, kv_len, q_off, scale=None):
    """Attention in 64 bits of q [T, Hq, D] over caches [blocks, 16, Hkv, D]: (out, lse, mean, most), where
    mean is sum w |v| / sum w, what a relative error of the weights moves an output by, and most the largest
    |scale| sum |q k| of a token's scores.  Rows that no request owns are NaN; block numbers outside the cache are left
    out.  A key or value that a token does not see has no part in its row, whatever it is."""
    T, Hq, D = q.shape
    Hkv = k_cache.shape[2]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    out, mean = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    lse, most = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    for i in range(len(kv_len)):
        q0, n, kv = int(q_off[i]), int(q_off[i + 1] - q_off[i]), int(kv_len[i])
        at = np.arange(kv)
        block = tables[i][at // BLOCK].astype(np.int64)
        good = (block >= 0) & (block < k_cache.shape[0])
        at, block = at[good], block[good]
        sees = at[None, :] <= (kv - n + np.arange(n))[:, None]             # [n, keys]
        for g in range(Hkv):
            k = k_cache[block, at % BLOCK, g].astype(np.float64)
            v = v_cache[block, at % BLOCK, g].astype(np.float64)
            for t in range(n) if n * at.size > 1 << 22 or not (np.isfinite(k).all() and np.isfinite(v).all()) else [None]:
                rows = slice(q0, q0 + n) if t is None else slice(q0 + t, q0 + t + 1)
                see = sees if t is None else sees[t:t + 1]
                if t is not None:                                          # only what it sees
                    kk, vv, see = k[see[0]], v[see[0]], see[:, see[0]]
                else:
                    kk, vv = k, v
                heads = slice(g * G, (g + 1) * G)
                x = q[rows, heads].astype(np.float64)                      # [r, G, D]
                with np.errstate(all="ignore"):
                    s = np.where(see[:, None, :], scale * (x @ kk.T), -np.inf)
                    top = s.max(-1, initial=-np.inf, keepdims=True)
                    w = np.where(see[:, None, :], np.exp(s - np.where(np.isneginf(top), 0, top)), 0)
                    total = w.sum(-1, keepdims=True)
                    none = total == 0
                    out[rows, heads] = np.where(none, 0, (w @ vv) / np.where(none, 1, total))
                    mean[rows, heads] = np.where(none, 0, (w @ np.abs(vv)) / np.where(none, 1, total))
                    lse[rows, heads] = np.where(none[..., 0], -np.inf, top[..., 0] + np.log(np.where(none, 1, total)[..., 0]))
                    most[rows, heads] = np.where(see[:, None, :], abs(scale) * (np.abs(x) @ np.abs(kk).T), 0).max(-1, initial=0)
    return out, lse, mean, most


# ------------------------------------------------------------------ a cache in 4 bits

SHARE = 32
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
EXPONENTS = {"bf16": (-125, 125), "fp16": (-23, 13)}


def fp4_encode(x, dtype):
    """(codes uint8 [..., 16 C], scales uint8 [..., C]) of values [..., D] in 64 bits: of each group of 32 the least power of
    two that 7 times holds the largest, and of each value the nearest magnitude, of two the one with the even code."""
    D = x.shape[-1]
    C = -(-D // SHARE)
    x = np.concatenate([np.asarray(x, np.float64), np.zeros((*x.shape[:-1], C * SHARE - D))], -1).reshape(*x.shape[:-1], C, SHARE)
    good = np.isfinite(x).all(-1)
    top = np.where(good, np.abs(np.where(np.isfinite(x), x, 0)).max(-1), 0)
    lo, hi = EXPONENTS[dtype]
    e = np.full(top.shape, hi)
    for k in range(hi - 1, lo - 1, -1):
        e = np.where(top <= 7 * 2.0 ** k, k, e)
    y = np.abs(np.where(np.isfinite(x), x, 0)) / 2.0 ** e[..., None]
    far = np.abs(y[..., None] - MAGNITUDES)
    nearest = far == far.min(-1, keepdims=True)
    even = nearest & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), nearest.argmax(-1)) + 8 * np.signbit(x)
    code = np.where(good[..., None], code, 0).reshape(*x.shape[:-2], C * SHARE).astype(np.uint8)
    return code[..., ::2] | code[..., 1::2] << 4, np.where(good, e + 127, 255).astype(np.uint8)


def fp4_decode(codes, scales, D):
    """The values [..., D] held, in 64 bits."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    x = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (x * np.repeat(power, SHARE, -1))[..., :D]
