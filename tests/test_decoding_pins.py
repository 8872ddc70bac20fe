"""Pins of oracle/decoding.py (CPU): closed forms, brute force, and the oracle of the causal reader where the definitions meet."""
import numpy as np
import pytest

from oracle import attention as oatt
from oracle import decoding as od


def _pool(rng, n, free, first):
    ids = rng.permutation(n).astype(np.int32)
    ring = np.full(n, -7, np.int32)
    ring[(first + np.arange(free)) % n] = ids[:free]
    return ring, ids[free:]


def test_steps_by_hand():
    """Blocks of 4.  Request 0 grows from 3 to 9 tokens, 1 gives 5 of 9 back, 2 ends but for its shared block, 3 starts."""
    tables = np.array([[10, -1, -1], [11, 12, 13], [14, 15, -1], [-1, -1, -1]], np.int32)
    pool = np.array([22, 23, -7, -7, -7, 20, 21], np.int32)            # a ring: 20, 21, 22, 23 from entry 5 on
    r = od.step_rows([3, 9, 8, 0], [6, -5, -8, 2], [0, 0, 1, 0], [5, 6, 7, 8], tables, pool, [5, 4], 4, 10, 30)
    assert r["tables"].tolist() == [[10, 20, 21], [11, 12, 13], [14, 15, -1], [22, -1, -1]]
    assert r["lengths"].tolist() == [9, 4, 0, 2] and r["offsets"].tolist() == [0, 6, 6, 6, 8]
    assert r["state"].tolist() == [1, 4, 8, 3, 3, 0]                   # 23 is left; 13, 12, 15 came back behind it
    assert r["pool"].tolist() == [22, 23, 13, 12, 15, 20, 21]
    assert r["pos"].tolist() == [3, 4, 5, 6, 7, 8, 0, 1, 0, 0] and r["seq"].tolist() == [0] * 6 + [3] * 2 + [-1] * 2
    assert r["slot"].tolist() == [43, 80, 81, 82, 83, 84, 88, 89, -1, -1] and r["aid"].tolist() == [5] * 6 + [8] * 2 + [-1] * 2


def test_steps_refuse_in_order():
    tables = np.full((4, 2), -1, np.int32)
    r = od.step_rows([0, 0, 0, 9], [4, 5, 1, 0], None, None, tables, np.arange(3, dtype=np.int32), [0, 3], 4, 100, 3)
    assert r["lengths"].tolist() == [4, 5, 0, 9] and r["state"].tolist()[2:] == [9, 3, 0, 2]     # no block left; a length past the table


@pytest.mark.parametrize("seed", range(4))
def test_steps_keep_every_block_once(seed):
    """Random growth and return: each block is in one table or in the pool, and rows land in their request's blocks."""
    rng = np.random.default_rng(seed)
    bs, seqs, blocks = int(rng.integers(1, 9)), 7, 60
    pool, _ = _pool(rng, blocks, blocks, int(rng.integers(0, blocks)))
    state, lengths, tables = np.array([np.flatnonzero(pool >= 0)[0], blocks], np.int32), np.zeros(seqs, np.int32), np.full((seqs, 12), -1, np.int32)
    first = int(rng.integers(0, blocks))
    pool, state = np.roll(pool, first - int(state[0])), np.array([first, blocks], np.int32)
    for _ in range(30):
        change = np.where(rng.random(seqs) < 0.4, -np.minimum(lengths, rng.integers(0, 40, seqs)), rng.integers(0, 30, seqs)).astype(np.int32)
        r = od.step_rows(lengths, change, None, None, tables, pool, state, bs, 64, blocks)
        tables, pool, lengths, state = r["tables"], r["pool"], r["lengths"], r["state"]
        used = [tables[s, b] for s in range(seqs) for b in range(-(-lengths[s] // bs))]
        free = [pool[(state[0] + i) % blocks] for i in range(state[1])]
        assert sorted(used + free) == list(range(blocks))
        for t in range(state[2]):
            s, p = r["seq"][t], r["pos"][t]
            assert r["slot"][t] == tables[s, p // bs] * bs + p % bs


def test_tree_rows_of_a_chain_and_of_roots():
    chain, pos = od.tree_rows(np.arange(-1, 69, dtype=np.int32), [0, 70], [5], 2)
    assert [int(m[0]) | int(m[1]) << 64 for m in chain] == [(1 << i + 1) - 1 for i in range(70)] and pos.tolist() == list(range(5, 75))
    roots, pos = od.tree_rows(np.full(3, -1, np.int32), [0, 3], [9], 1)
    assert roots[:, 0].tolist() == [1, 2, 4] and pos.tolist() == [9, 9, 9]
    bad, pos = od.tree_rows(np.array([-1, 1, 1, 0, -3], np.int32), [0, 5], [2], 1)      # its own parent, its child, a fine one, no place
    assert bad[:, 0].tolist() == [1, 0, 0, 9, 0] and pos.tolist() == [2, 2, 2, 3, 2]


def _cache(rng, lens, bs, hkv, d):
    n = [-(-x // bs) for x in lens]
    perm = rng.permutation(sum(n) + 2).astype(np.int32)
    tables, at = np.full((len(lens), max(n) + 1), -1, np.int32), 0
    for s, m in enumerate(n):
        tables[s, :m] = perm[at: at + m]
        at += m
    return tables, *(rng.standard_normal((len(perm) * bs, hkv * d)) for _ in range(2))


def test_a_chain_is_the_causal_reader():
    rng = np.random.default_rng(3)
    ctx, n, bs, hq, hkv, d = [7, 0, 20], [3, 4, 1], 4, 4, 2, 8
    tables, k, v = _cache(rng, [c + m for c, m in zip(ctx, n)], bs, hkv, d)
    off = np.concatenate([[0], np.cumsum(n)])
    parents = np.concatenate([np.arange(-1, m - 1) for m in n])
    mask, pos = od.tree_rows(parents, off, ctx, 1)
    q = rng.standard_normal((8, hq * d))
    want = oatt.paged_attention(q, k, v, tables, np.repeat(np.arange(3), n), pos, bs, hq, hkv, d)
    assert np.allclose(od.tree_attention(q, k, v, tables, off, ctx, mask, bs, hq, hkv, d), want, rtol=1e-13)


def test_a_path_of_a_tree_is_its_own_sequence():
    """A leaf's row equals the last row of a sequence that holds its path alone; other branches may hold anything."""
    rng = np.random.default_rng(4)
    bs, hq, hkv, d, c = 4, 2, 1, 8, 6
    parents = np.array([-1, 0, 0, 2, 1, 3], np.int32)
    tables, k, v = _cache(rng, [c + 6], bs, hkv, d)
    mask, pos = od.tree_rows(parents, [0, 6], [c], 1)
    assert pos.tolist() == [6, 7, 7, 8, 8, 9]
    slot = [int(tables[0, p // bs]) * bs + p % bs for p in range(c + 6)]
    for j in (1, 4):
        k[slot[c + j]] = v[slot[c + j]] = np.nan
    q = rng.standard_normal((6, hq * d))
    got = od.tree_attention(q, k, v, tables, [0, 6], [c], mask, bs, hq, hkv, d)[5]
    path = [*range(c), c, c + 2, c + 3, c + 5]
    k2, v2 = (np.stack([x[slot[p]] for p in path] + [x[slot[0]] * 0] * 2) for x in (k, v))
    want = oatt.paged_attention(q[5:], k2, v2, np.array([[0, 1, 2]]), [0], [9], bs, hq, hkv, d)
    assert np.allclose(got, want[0], rtol=1e-13)


def test_bounds_enclose_the_keys_and_their_scores():
    """Bounds times scale enclose every key up to fp32 rounding, touch the largest component, and the score (with q on its 8-bit grid) bounds the heads' sum of scores."""
    rng = np.random.default_rng(5)
    bs, hq, hkv, d = 4, 4, 2, 16
    k = rng.standard_normal((12 * bs, hkv * d)) * np.exp(rng.standard_normal((12 * bs, 1)))
    bounds, scales = od.block_bounds(k, np.arange(12 * bs), np.zeros((12, hkv, 2, d), np.int8), np.zeros((12, hkv), np.float32), bs, hkv, d)
    keys = k.reshape(12, bs, hkv, d)
    assert np.all(bounds[:, :, 0] * scales[..., None] >= keys.max(1) * (1 - 1e-6) - 1e-6) and np.all(bounds[:, :, 1] * scales[..., None] <= keys.min(1) + 1e-6)
    assert np.all(np.abs(bounds.astype(int)).max((2, 3)) == 127)
    q = rng.integers(-31, 32, (1, hq * d)).astype(float)
    q[0, 0: 2 * d: d], q[0, 2 * d:: d] = 63, 64                        # largest sums: 126 and 128, so that head 0's grid is not 1
    for h in range(hkv):
        x = q.reshape(hkv, 2, d)[h]
        both = np.concatenate([np.maximum(x, 0).sum(0), np.minimum(x, 0).sum(0)])
        step = np.abs(both).max() / 127
        score = np.array(od.block_scores(q[0], bounds, scales, range(12), h, hq, hkv, d)) * step
        real = np.einsum("gd,nbd->nbg", x, keys[:, :, h]).sum(-1).max(1)
        slack = step / 2 * 2 * d * np.abs(keys[:, :, h]).max((1, 2))   # q's rounding
        assert np.all(score >= real - slack - 1e-3)


def test_bounds_of_part_of_a_block_and_of_values_that_are_not_finite():
    k = np.array([[1.0, -2], [3, 4], [np.nan, 9], [9, 9]])
    start = np.zeros((1, 1, 2, 2), np.int8), np.zeros((1, 1), np.float32)
    b, s = od.block_bounds(k, [0, 1], *start, 4, 1, 2)
    assert b[0, 0].tolist() == [[96, 127], [31, -64]] and s[0, 0] == np.float32(4) / np.float32(127)
    b, s = od.block_bounds(k, [0, 1, 2], *start, 4, 1, 2)
    assert not b.any() and np.isinf(s[0, 0])
    b, s = od.block_bounds(k, [-1, 4, 7], *start, 4, 1, 2)
    assert not b.any() and not s.any()


def test_selection_by_hand():
    """One head of two components, q = (1, 0): a block's score is scale times 127 times its upper bound."""
    bounds = np.zeros((8, 1, 2, 2), np.int8)
    bounds[:, 0, 0, 0] = [10, 50, 50, 20, 90, 50, 1, 2]
    scales = np.ones((8, 1), np.float32)
    tables = np.arange(8, dtype=np.int32)[None]
    pick = lambda budget, first, recent, pos=31: od.block_select(np.array([[1.0, 0]]), bounds, scales, tables, [0], [pos], 4, budget, first, recent, 1, 1, 2)[0, 0].tolist()
    assert pick(3, 0, 1) == [1, 4, 7] and pick(4, 0, 1) == [1, 2, 4, 7] and pick(4, 1, 2) == [0, 4, 6, 7]
    assert pick(9, 1, 1) == [*range(8), -1] and pick(3, 1, 1, 5) == [0, 1, -1]
    scales[3] = np.inf
    assert pick(2, 0, 1) == [3, 7]
    tables[0, 3] = 8                                                    # outside the cache
    assert pick(2, 0, 1) == [4, 7]


def test_all_blocks_selected_is_the_whole_context():
    rng = np.random.default_rng(6)
    bs, hq, hkv, d = 5, 4, 2, 8
    tables, k, v = _cache(rng, [23, 9], bs, hkv, d)
    seq, pos, q = np.array([0, 0, 1]), np.array([22, 14, 8]), rng.standard_normal((3, hq * d))
    want = oatt.paged_attention(q, k, v, tables, seq, pos, bs, hq, hkv, d)
    every = np.broadcast_to(np.arange(6, dtype=np.int32), (3, hkv, 6))
    assert np.allclose(od.selected_attention(q, k, v, tables, seq, pos, every, bs, hq, hkv, d), want, rtol=1e-13)
    twice = np.broadcast_to(np.array([-1, 0, 0, 1, 1, 2, 3, 4, 99, 5], np.int32), (3, hkv, 10))
    assert np.allclose(od.selected_attention(q, k, v, tables, seq, pos, twice, bs, hq, hkv, d), want, rtol=1e-13)
