"""Oracle for steps built from lengths, drafted trees and contexts read in part (include/alora_steps.h, alora_tree.h, alora_select.h).

TEST INFRASTRUCTURE ONLY: plain Python and numpy in fp64, the definitions written out one request, row and head at a time; the GPU code shares
nothing with it.
"""
from __future__ import annotations

import numpy as np


def step_rows(lengths, change, kept, adapters, tables, pool, state, block_size, row_cap, n_blocks):
    """Serves the requests in their order; returns a dict of everything alora_step_rows writes (tables and pool as copies)."""
    tables, pool = tables.copy(), pool.copy()
    n_seqs, max_blocks = tables.shape
    ring, cap = len(pool), min(max_blocks * block_size, 2**31 - 1)
    first, count = int(state[0]), int(state[1])
    if not (0 <= first < ring and 0 <= count <= ring):
        first = count = 0
    blocks_of = lambda n: -(-n // block_size)
    rows, offsets, lengths_out = [], [0], []
    returned, taken, refused, out_of_room = [], 0, 0, False
    asked_blocks = asked_rows = 0
    for s in range(n_seqs):
        n, c = int(lengths[s]), int(change[s])
        ok = 0 <= n <= cap and 0 <= n + c <= cap
        if ok and c > 0:
            asked_blocks += blocks_of(n + c) - blocks_of(n)
            asked_rows += c
            out_of_room = out_of_room or asked_blocks > count or asked_rows > row_cap
            ok = not out_of_room
        if not ok:
            refused += 1
            lengths_out.append(n)
            offsets.append(len(rows))
            continue
        for b in range(blocks_of(n), blocks_of(n + c)):
            tables[s, b] = pool[(first + taken) % ring]
            taken += 1
        for b in range(blocks_of(n) - 1, max(blocks_of(n + c), 0 if kept is None else int(kept[s])) - 1, -1):
            returned.append(int(tables[s, b]))
        for p in range(n, n + c):
            block = int(tables[s, p // block_size])
            rows.append((s, p, -1 if adapters is None else int(adapters[s]), block * block_size + p % block_size if 0 <= block < n_blocks else -1))
        lengths_out.append(n + c)
        offsets.append(len(rows))
    returned = returned[: ring - count]
    for i, b in enumerate(returned):
        pool[(first + count + i) % ring] = b
    n_rows = len(rows)
    rows += [(-1, 0, -1, -1)] * (row_cap - n_rows)
    cols = list(zip(*rows)) if rows else [()] * 4
    return dict(tables=tables, pool=pool, lengths=np.array(lengths_out, np.int32), offsets=np.array(offsets, np.int32),
                state=np.array([(first + taken) % ring if ring else 0, count - taken + len(returned), n_rows, taken, len(returned), refused], np.int32),
                seq=np.array(cols[0], np.int32), pos=np.array(cols[1], np.int32), aid=np.array(cols[2], np.int32), slot=np.array(cols[3], np.int64))


def tree_rows(parents, offsets, context, words):
    """(mask uint64 [rows, words], positions)"""
    rows = len(parents)
    mask, pos = np.zeros((rows, words), np.uint64), np.zeros(rows, np.int32)
    for s in range(len(context)):
        a, b = int(offsets[s]), int(offsets[s + 1])
        seen = []
        for i in range(b - a):
            p = int(parents[a + i])
            line = None
            if i < 64 * words and -1 <= p < i:
                line = [i] if p == -1 else None if seen[p] is None else [*seen[p], i]
            seen.append(line)
            pos[a + i] = int(context[s]) + (len(line) - 1 if line else 0)
            for j in line or []:
                mask[a + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return mask, pos


def _slot(table, place, block_size, n_blocks):
    block = int(table[place // block_size])
    return block * block_size + place % block_size if 0 <= block < n_blocks else -1


def attend(q, k_cache, v_cache, slots, hq, hkv, d, scale=None):
    """One row's attention over the cache slots given for each K/V head: [hq * d]"""
    scale = 1.0 / np.sqrt(float(d)) if scale is None else scale
    out = np.zeros(hq * d)
    for h in range(hq):
        g = h // (hq // hkv)
        at = np.array([s for s in slots[g] if s >= 0], np.int64)
        if not len(at):
            continue
        score = scale * (k_cache[at].reshape(len(at), hkv, d)[:, g] @ q[h * d:(h + 1) * d])
        w = np.exp(score - score.max())
        out[h * d:(h + 1) * d] = (w / w.sum()) @ v_cache[at].reshape(len(at), hkv, d)[:, g]
    return out


def tree_attention(q, k_cache, v_cache, tables, offsets, context, mask, block_size, hq, hkv, d, scale=None):
    out = np.zeros((q.shape[0], hq * d))
    n_blocks, cap = k_cache.shape[0] // block_size, tables.shape[1] * block_size
    for s in range(len(context)):
        a, b, c = int(offsets[s]), int(offsets[s + 1]), min(int(context[s]), cap)
        for t in range(a, b):
            bits = [j for j in range(min(b - a, 64 * mask.shape[1])) if int(mask[t, j // 64]) >> (j % 64) & 1 and c + j < cap]
            slots = [_slot(tables[s], p, block_size, n_blocks) for p in [*range(c), *(c + j for j in bits)]]
            out[t] = attend(q[t], k_cache, v_cache, [slots] * hkv, hq, hkv, d, scale)
    return out


TINY = 2.0 ** -100


def _factor(a):
    """127 / a in fp32, as the definition has it."""
    return np.float32(127) / np.float32(a) if TINY <= a < np.inf else np.float32(0)


def block_bounds(k_cache, slots, bounds, scales, block_size, hkv, d):
    """Copies of bounds [blocks, hkv, 2, d] and scales with the blocks of `slots` renewed."""
    bounds, scales = bounds.copy(), scales.copy()
    n_slots = bounds.shape[0] * block_size
    for i, slot in enumerate(int(x) for x in slots):
        if not 0 <= slot < n_slots:
            continue
        later = [int(x) for x in slots[i + 1:] if 0 <= int(x) < n_slots]
        if later and later[0] // block_size == slot // block_size:
            continue
        b, off = divmod(slot, block_size)
        k = k_cache[b * block_size: b * block_size + off + 1].reshape(off + 1, hkv, d)
        for h in range(hkv):
            a = np.abs(k[:, h]).max()
            if not np.isfinite(a):
                bounds[b, h], scales[b, h] = 0, np.inf
                continue
            f = _factor(a)
            bounds[b, h, 0] = np.clip(np.ceil(k[:, h].max(0).astype(np.float32) * f), -127, 127)
            bounds[b, h, 1] = np.clip(np.floor(k[:, h].min(0).astype(np.float32) * f), -127, 127)
            scales[b, h] = np.float32(a) / np.float32(127)
    return bounds, scales


def block_scores(q, bounds, scales, blocks, h, hq, hkv, d):
    """Scores of the given blocks for one row and K/V head; minus infinity for blocks outside the cache."""
    g = hq // hkv
    x = q.reshape(hkv, g, d)[h]
    both = np.concatenate([np.maximum(x, 0).sum(0), np.minimum(x, 0).sum(0)]).astype(np.float32)
    f = _factor(float(np.abs(both).max()))
    whole = np.rint(both * f).astype(np.int64)
    largest = np.finfo(np.float32).max
    out = []
    for b in blocks:
        if not 0 <= b < bounds.shape[0]:
            out.append(-np.inf)
        elif not np.isfinite(scales[b, h]):
            out.append(float(largest))
        else:
            with np.errstate(over="ignore"):
                out.append(float(np.clip(np.float32(int(whole @ bounds[b, h].reshape(-1).astype(np.int64))) * np.float32(scales[b, h]), -largest, largest)))
    return out


def block_select(q, bounds, scales, tables, seq, pos, block_size, budget, n_first, n_recent, hq, hkv, d):
    out = np.full((len(seq), hkv, budget), -1, np.int32)
    for t in range(len(seq)):
        if not (0 <= seq[t] < tables.shape[0] and pos[t] >= 0):
            continue
        n = min(int(pos[t]) // block_size + 1, tables.shape[1])
        for h in range(hkv):
            always = [b for b in range(n) if b < n_first or b >= n - n_recent]
            rest = [b for b in range(n) if b not in set(always)]
            score = block_scores(q[t], bounds, scales, [int(tables[seq[t], b]) for b in rest], h, hq, hkv, d)
            best = [b for _, b in sorted(zip([-x for x in score], rest))]
            chosen = sorted(always + best)[:n] if n <= budget else sorted(always + best[: budget - len(always)])
            out[t, h, : len(chosen)] = chosen
    return out


def selected_attention(q, k_cache, v_cache, tables, seq, pos, selected, block_size, hq, hkv, d, scale=None):
    out = np.zeros((q.shape[0], hq * d))
    n_blocks = k_cache.shape[0] // block_size
    for t in range(q.shape[0]):
        if not (0 <= seq[t] < tables.shape[0] and pos[t] >= 0):
            continue
        p, n = int(pos[t]), min(int(pos[t]) // block_size + 1, tables.shape[1])
        lists = []
        for h in range(hkv):
            e = [int(x) for x in selected[t, h]]
            use = [b for i, b in enumerate(e) if 0 <= b < n and (i == 0 or b > e[i - 1])]
            lists.append([_slot(tables[seq[t]], j, block_size, n_blocks) for b in use for j in range(b * block_size, (b + 1) * block_size) if j <= p])
        out[t] = attend(q[t], k_cache, v_cache, lists, hq, hkv, d, scale)
    return out
