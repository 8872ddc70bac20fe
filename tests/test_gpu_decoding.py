"""GPU parity of steps built from lengths, drafted trees and selected blocks (alora_steps.h, alora_tree.h, alora_select.h) against oracle/decoding.py.

Whole numbers have to be equal.  Attention, per element, from the roundings made (u = 2^-24): a score is a sum of head_dim products, off by
head_dim u S at most, S = scale * sum_d |q_d| max_j |k_jd|; a weight by twice that (its own score's and the largest one's) and a few u of the power and of
the sums, together (2 head_dim S + 64) u of A = sum_j w_j |v_j|, which the oracle gives for |v|; in bf16 the weights are rounded for the product
with V, half a step (2^-8) of A, and the result is rounded once, half a step of its value."""
import numpy as np
import pytest
import torch

from oracle import decoding as od
from paper_2512_17910_amd import binding as ab
from gpu_util import raw_bits, to_f64

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def values(rng, shape, dt, std=1.0):
    return dev((rng.standard_normal(shape) * std).astype(np.float32)).to(dt)


# ---- steps ----------------------------------------------------------------------------------------
class Step:
    """A call's tensors on the device and what the oracle makes of them."""

    def __init__(self, lengths, change, kept, adapters, tables, pool, state, bs, row_cap, n_blocks):
        i32 = lambda x: None if x is None else np.asarray(x, np.int32)
        self.host = [i32(x) for x in (lengths, change, kept, adapters, tables, pool, state)]
        self.bs, self.row_cap, self.n_blocks = bs, row_cap, n_blocks
        self.dev = [None if x is None else dev(x) for x in self.host]
        n = len(lengths)
        new = lambda k, dt=torch.int32: torch.full((k,), -99, dtype=dt, device="cuda")
        self.out = [new(n), new(6), new(n + 1), new(row_cap), new(row_cap), new(row_cap), new(row_cap, torch.int64)]
        self.dims = ab.make_step_dims(self.dev[4], bs, row_cap, self.dev[5], n_blocks * bs)

    def run(self):
        ab.alora_step_rows(*self.dev, *self.out, self.dims)

    def check(self, want=None):
        want = want or od.step_rows(*self.host, self.bs, self.row_cap, self.n_blocks)
        got = [*self.dev[4:6], *self.out]
        for x, name in zip(got, ("tables", "pool", "lengths", "state", "offsets", "seq", "pos", "aid", "slot")):
            assert np.array_equal(x.cpu().numpy(), want[name]), (name, x.cpu().numpy(), want[name])
        return want


def step_case(rng, n_seqs, bs, most, max_blocks, spare, kept=True, adapters=True, pad=0):
    cap = max_blocks * bs
    lengths = rng.integers(0, max(1, cap - most) + 1, n_seqs)
    change = np.where(rng.random(n_seqs) < 0.3, -np.minimum(lengths, rng.integers(0, cap + 1, n_seqs)), rng.integers(0, most + 1, n_seqs))
    have = -(-lengths // bs)
    need = int(np.maximum(-(-(lengths + change) // bs) - have, 0).sum())
    blocks = int(have.sum()) + max(0, need + spare) + 3
    perm = rng.permutation(blocks).astype(np.int32)
    tables = np.full((n_seqs, max_blocks), -5, np.int32)
    at = np.arange(max_blocks)[None] < have[:, None]
    tables[at] = perm[: have.sum()]
    first, free = int(rng.integers(0, blocks)), max(0, need + spare)
    pool = np.full(blocks, -6, np.int32)
    pool[(first + np.arange(free)) % blocks] = perm[have.sum(): have.sum() + free]
    return Step(lengths, change, rng.integers(0, 3, n_seqs) if kept else None, rng.integers(-1, 9, n_seqs) if adapters else None, tables, pool,
                [first, free, 0, 0, 0, 0], bs, int(np.maximum(change, 0).sum()) + pad, blocks)


@pytest.mark.parametrize("n_seqs,bs,most,max_blocks", [(1, 16, 1, 4), (1, 1, 5, 40), (7, 5, 9, 11), (255, 16, 1, 9), (256, 16, 33, 9), (257, 3, 20, 30), (700, 16, 64, 20),
                                                       (3, 16, 5000, 400), (90, 7, 900, 300)])
@pytest.mark.parametrize("spare,pad", [(5, 0), (0, 13), (-3, 0), (-40, 700)])
def test_steps(n_seqs, bs, most, max_blocks, spare, pad):
    rng = np.random.default_rng(n_seqs * 31 + bs + most + spare + 40)
    s = step_case(rng, n_seqs, bs, most, max_blocks, spare, kept=spare != 0, adapters=pad != 13, pad=pad)
    s.run()
    want = s.check()
    s.run()                                                            # the same inputs again: the same results
    s.check(want)


def test_steps_without_room_for_rows():
    rng = np.random.default_rng(1)
    s = step_case(rng, 300, 16, 8, 10, 5)
    for cap in (0, 1, 500):
        t = Step(*s.host, s.bs, cap, s.n_blocks)
        t.run()
        assert t.check()["state"][5] > 0


def test_steps_of_no_requests_and_of_no_pool():
    s = Step([], [], None, None, np.zeros((0, 3)), [4, 5], [1, 1, 0, 0, 0, 0], 16, 5, 9)
    s.run()
    s.check()
    s = Step([3, 16, 0], [13, 1, 0], None, None, np.array([[1], [2], [3]]), [], [0, 0, 0, 0, 0, 0], 16, 20, 9)
    s.run()
    assert s.check()["state"].tolist() == [0, 0, 13, 0, 0, 1]


def test_steps_with_lengths_and_pools_out_of_range():
    n = 2 ** 31 - 1
    tables = np.array([[0, 1, 77], [2, 3, 4], [5, -1, -1], [6, 7, 8], [9, 10, 11]], np.int32)
    for state in ([2, 4], [-1, 4], [2, 9], [7, 1]):
        s = Step([33, -4, 5, n, 40], [10, 8, 20, n, -n], None, None, tables, [12, 99, 13, -8, 14, 15, 16], [*state, 0, 0, 0, 0], 16, 50, 17)
        s.run()
        s.check()


def test_steps_of_lengths_up_to_the_largest():
    """A length that, rounded up to blocks, passes 31 bits; the table has room for exactly so many."""
    n, bs, columns = 2 ** 31 - 5, 16, 1 << 27
    tables = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    last = (n - 1) // bs
    tables[0, last - 40: last + 1] = torch.arange(100, 141, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pool = i32(*range(60))
    for change, length, freed in ((3, n + 3, []), (4, n + 4, []), (5, n, []), (-500, n - 500, [140 - i for i in range(31)])):
        out = [i32(*[-9] * k) for k in (1, 6, 2, 8, 8, 8)] + [torch.full((8,), -9, dtype=torch.int64, device="cuda")]
        ab.alora_step_rows(i32(n), i32(change), None, None, tables, pool, i32(7, 2, 0, 0, 0, 0), *out, ab.make_step_dims(tables, bs, 8, pool, 200 * bs))
        served = length - n if 0 < length - n else 0
        assert out[0].item() == length and out[1].tolist() == [7, 2 + len(freed), served, 0, len(freed), int(change == 5)]
        assert out[4].tolist() == [*range(n, n + served), *[0] * (8 - served)]
        assert out[6].tolist() == [140 * bs + (n + i) % bs for i in range(served)] + [-1] * (8 - served)
        assert pool[9: 9 + len(freed)].tolist() == freed


def test_steps_that_give_back_more_blocks_than_a_pool_holds():
    """2^30 blocks of one position and more: the sums stop there, the pool much earlier."""
    columns = (1 << 30) + 100
    tables = torch.empty((2, columns), dtype=torch.int32, device="cuda")
    tables[0, :100] = torch.arange(100, dtype=torch.int32, device="cuda")
    tables[1, -300:] = torch.arange(1000, 1300, dtype=torch.int32, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pool = torch.full((300,), -6, dtype=torch.int32, device="cuda")
    out = [i32(*[-9] * k) for k in (2, 6, 3, 1, 1, 1)] + [torch.full((1,), -9, dtype=torch.int64, device="cuda")]
    ab.alora_step_rows(i32(100, columns), i32(-100, -columns), None, None, tables, pool, i32(290, 0, 0, 0, 0, 0), *out, ab.make_step_dims(tables, 1, 1, pool, 5000))
    assert out[0].tolist() == [0, 0] and out[1].tolist() == [290, 300, 0, 0, 300, 0]
    assert torch.cat([pool[290:], pool[:290]]).tolist() == [*range(99, -1, -1), *range(1299, 1099, -1)]


def test_a_loop_of_steps_on_the_device():
    """Lengths, tables and pool stay on the device over 40 steps; the loop exchanges the states."""
    rng = np.random.default_rng(8)
    n, bs, blocks = 19, 4, 150
    s = Step(np.zeros(n), np.zeros(n), None, None, np.full((n, 20), -1), rng.permutation(blocks), [0, blocks, 0, 0, 0, 0], bs, 120, blocks)
    tables, pool, lengths, state = s.host[4], s.host[5], s.host[0], s.host[6]
    a, b = (s.dev[0], s.dev[6]), (s.out[0], s.out[1])
    for i in range(40):
        change = np.where(rng.random(n) < 0.3, -rng.integers(0, 30, n), rng.integers(0, 12, n)).astype(np.int32)      # (some give back more than they have: refused)
        s.dev[1].copy_(torch.from_numpy(change))
        ab.alora_step_rows(a[0], s.dev[1], None, None, s.dev[4], s.dev[5], a[1], *b, *s.out[2:], s.dims)
        w = od.step_rows(lengths, change, None, None, tables, pool, state, bs, 120, blocks)
        tables, pool, lengths, state = w["tables"], w["pool"], w["lengths"], w["state"]
        for x, name in zip((s.dev[4], s.dev[5], *b, *s.out[2:]), ("tables", "pool", "lengths", "state", "offsets", "seq", "pos", "aid", "slot")):
            assert np.array_equal(x.cpu().numpy(), w[name]), (i, name)
        a, b = b, a


# ---- trees ----------------------------------------------------------------------------------------
def offsets_of(n, first=0):
    return (first + np.concatenate([[0], np.cumsum(n)])).astype(np.int32)


def parents_of(rng, n):
    return np.concatenate([[int(rng.integers(-1, i)) if rng.random() < 0.5 else i - 1 for i in range(m)] for m in n] or [[]]).astype(np.int32)


@pytest.mark.parametrize("words", [1, 2, 3, 4])
@pytest.mark.parametrize("n", [[1], [0, 5, 64, 0], [63, 1, 65, 200], [300, 2], [2] * 300], ids=["one", "empty", "wide", "too-wide", "many"])
def test_tree_rows(words, n):
    rng = np.random.default_rng(words + len(n))
    for bad, chain in ((0.0, False), (0.1, False), (0.0, True)):
        parents = np.concatenate([np.arange(-1, m - 1) for m in n]).astype(np.int32) if chain else parents_of(rng, n)
        spoil = rng.random(len(parents)) < bad
        parents[spoil] = rng.choice([-2, 500, 2 ** 31 - 1, -2 ** 31], int(spoil.sum()))
        before, behind = 3 * (bad > 0), 5 * (bad > 0)                  # rows of no sequence
        parents, off = np.concatenate([np.zeros(before, np.int32), parents, np.zeros(behind, np.int32)]).astype(np.int32), offsets_of(n, before)
        ctx = rng.integers(0, 9000, len(n)).astype(np.int32)
        mask, pos = torch.full((len(parents), words), -1, dtype=torch.int64, device="cuda"), torch.full((len(parents),), -1, dtype=torch.int32, device="cuda")
        ab.alora_tree_rows(dev(parents), dev(off), dev(ctx), mask, pos)
        wm, wp = od.tree_rows(parents, off, ctx, words)
        assert np.array_equal(mask.cpu().numpy().view(np.uint64), wm) and np.array_equal(pos.cpu().numpy(), wp)


class Cache:
    """A pool whose slots outside the sequences' lengths hold NaN."""

    def __init__(self, rng, lens, dt, hkv, d, bs, std=1.0, more_columns=1):
        n = [-(-int(x) // bs) for x in lens]
        perm = rng.permutation(sum(n) + 3).astype(np.int32)
        self.tables, at = np.full((len(lens), max([*n, 0]) + more_columns), -1, np.int32), 0
        used = np.zeros(len(perm) * bs, bool)
        for s, m in enumerate(n):
            self.tables[s, :m] = perm[at: at + m]
            p = np.arange(int(lens[s]))
            used[self.tables[s, p // bs] * bs + p % bs] = True
            at += m
        self.k, self.v = (values(rng, (len(used), hkv * d), dt, std) for _ in range(2))
        self.k[dev(~used)] = float("nan")
        self.v[dev(~used)] = float("nan")


def close(got, q, k, v, scale, hq, hkv, d, dt, attention):
    """attention(v): the oracle's rows for these values; see the top."""
    got, want, size = to_f64(got), attention(v), attention(np.abs(v))
    assert np.isfinite(got).all()
    kmax = np.nan_to_num(np.abs(k), nan=0.0, posinf=0.0).max(0).reshape(hkv, d)
    S = scale * (np.abs(q).reshape(-1, hkv, hq // hkv, d) * kmax[None, :, None]).sum(-1).reshape(-1, hq, 1)
    rel = (2 * d * S + 64) * U32 + (HALF[dt] if dt == torch.bfloat16 else 0.0)
    err = (rel * size.reshape(-1, hq, d)).reshape(size.shape)
    over = np.abs(got - want) - (HALF[dt] * (np.abs(want) + err) + err)
    assert np.all(over <= 0), (float(over.max()), np.unravel_index(int(np.argmax(over)), over.shape))


class Tree:
    def __init__(self, dtype, ctx, n, words, hq, hkv, d, bs, seed=0, random_masks=False, first=0, behind=0, std=1.0, scale=0.0):
        rng = self.rng = np.random.default_rng(seed)
        self.dt, self.ctx, self.n, self.words, self.sizes, self.bs, self.scale = DT[dtype], np.array(ctx, np.int32), n, words, (hq, hkv, d), bs, scale
        self.off = offsets_of(n, first)
        rows = int(self.off[-1]) + behind
        self.cache = Cache(rng, self.ctx + np.array(n), self.dt, hkv, d, bs, std)
        if random_masks:
            self.mask = rng.integers(0, 2 ** 63, (rows, words), dtype=np.uint64) & rng.integers(0, 2 ** 63, (rows, words), dtype=np.uint64)
            self.mask[rng.random(rows) < 0.2] = 0
        else:
            self.mask = np.zeros((rows, words), np.uint64)
            self.mask[first: self.off[-1]] = od.tree_rows(parents_of(rng, n), offsets_of(n), self.ctx, words)[0]
        self.q = values(rng, (rows, hq * d), self.dt)
        self.out = torch.full_like(self.q, float("nan"))
        self.bt, self.dev = dev(self.cache.tables), [dev(self.off), dev(self.ctx), dev(self.mask.view(np.int64))]
        self.dims = ab.make_attn_dims(self.q, self.cache.k, self.bt, hq, hkv, d, bs, scale)
        self.ws = torch.full((ab.alora_tree_attention_workspace_bytes(self.dims, words) // 4 + 4,), float("nan"), device="cuda")

    def run(self):
        ab.alora_tree_attention(self.q, self.cache.k, self.cache.v, self.bt, *self.dev, self.out, self.dims, self.ws)
        torch.cuda.synchronize()
        return self.out

    def check(self):
        hq, hkv, d = self.sizes
        q, k, v = to_f64(self.q), to_f64(self.cache.k), to_f64(self.cache.v)
        scale = self.scale or d ** -0.5
        close(self.out, q, k, v, scale, hq, hkv, d, self.dt,
              lambda v: od.tree_attention(q, k, v, self.cache.tables, self.off, self.ctx, self.mask, self.bs, hq, hkv, d, scale))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("bs", [16, 5])
def test_tree_attention(dtype, d, group, bs):
    """Ragged contexts, one of them empty; trees from one draft to more than a tile of rows; a sequence without drafts."""
    t = Tree(dtype, [0, 33, 270, 1, 95, 600], [7, 1, 40, 0, 64, 3], 1, 2 * group, 2, d, bs, seed=d + group + bs)
    print("tree", dtype, d, group, bs, flush=True)
    t.run()
    t.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("words,n", [(2, [100, 3]), (3, [192, 0, 1]), (4, [256, 129]), (4, [31]), (1, [90, 2])])
def test_wide_trees_and_any_masks(dtype, words, n):
    """Masks that are no tree's, some empty (over a context of nothing: a row of zeros), rows in front of and behind all sequences, drafts that the masks have no
    room for."""
    t = Tree(dtype, [0, 40, 17][: len(n)], n, words, 4, 1, 128, 16, seed=words, random_masks=True, first=3, behind=9)
    t.run()
    t.check()
    got = to_f64(t.out)
    assert not got[:3].any() and not got[-9:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences_and_few(dtype):
    rng = np.random.default_rng(2)
    ctx = rng.integers(0, 50, 300)
    ctx[[5, 270]] = 1500
    for c, n, hkv in ((ctx, rng.integers(0, 4, 300).tolist(), 1), ([9000], [1], 2), ([5000, 20], [17, 2], 8), ([2047, 2048, 2049, 4097], [1, 1, 1, 1], 1)):
        t = Tree(dtype, c, n, 1, 4 * hkv, hkv, 64, 16, seed=3)
        print("tree", dtype, len(c), flush=True)
        t.run()
        t.check()
        first = raw_bits(t.out).copy()
        t.ws.fill_(1e30)
        t.out.fill_(float("nan"))
        assert np.array_equal(raw_bits(t.run()), first)                # whatever the workspace held


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs", [64, 65, 257, 513, 1100])
@pytest.mark.parametrize("most", [3, 9])
def test_more_sequences_than_a_wavefront_or_a_workgroup_looks_at(dtype, seqs, most):
    """Ragged, some without a context, some without drafts; two are long, one of them with many rows: their parts and tiles are written by many threads."""
    rng = np.random.default_rng(seqs + most)
    ctx, n = rng.integers(0, 40, seqs), rng.integers(0, most + 1, seqs)
    ctx[[7, seqs - 2]], n[seqs - 2] = (1900, 900), 130
    t = Tree(dtype, ctx, n.tolist(), 3, 4, 1, 64, 16, seed=seqs, first=2, behind=3)
    t.ws[ab.alora_tree_attention_workspace_bytes(t.dims, 3) // 4:] = 7.0
    t.run()
    assert (t.ws[ab.alora_tree_attention_workspace_bytes(t.dims, 3) // 4:] == 7.0).all()
    t.check()
    first = raw_bits(t.out).copy()
    t.ws.fill_(-1e30)
    t.out.fill_(float("nan"))
    assert np.array_equal(raw_bits(t.run()), first)


def test_parts_of_many_ragged_sequences_have_room():
    """Contexts of all lengths over several turns of the chip: whole tiles and parts side by side, in a workspace that has room for few of them."""
    rng = np.random.default_rng(17)
    for seqs, hkv, longest in ((40, 8, 3000), (63, 8, 9000), (150, 8, 4000), (90, 2, 20000)):
        ctx = (longest * rng.random(seqs) ** 3).astype(int)
        t = Tree("bf16", ctx, rng.integers(1, 12, seqs).tolist(), 1, 2 * hkv, hkv, 64, 16, seed=18)
        need = ab.alora_tree_attention_workspace_bytes(t.dims, 1) // 4
        t.ws[need:] = 7.0
        t.run()
        assert (t.ws[need:] == 7.0).all()
        t.check()


def test_peaked_scores_and_scale():
    for scale in (0.0, 0.3):
        t = Tree("bf16", [300, 20], [20, 30], 1, 8, 2, 128, 16, seed=4, std=6.0, scale=scale)
        t.run()
        t.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq", [2, 8])                                 # (with two, wavefronts share the columns)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_drafts_that_a_row_does_not_see_may_hold_anything(dtype, hq, bad):
    """Two branches; the second one's keys and values are not finite.  Rows of the first are as if it were not there."""
    def branches(value):
        t = Tree(dtype, [70, 5], [41, 1], 1, hq, 2, 128, 16, seed=5)
        left = np.zeros(42, bool)
        left[1: 41: 2] = True
        for i in range(41):
            same = np.arange(41) % 2 == i % 2
            t.mask[i, 0] = sum(1 << int(j) for j in range(i + 1) if same[j] or j == 0)
        t.mask[:41] &= np.uint64((1 << 41) - 1)
        t.dev[2].copy_(dev(t.mask.view(np.int64)))
        p = 70 + np.flatnonzero(left[:41])
        slot = dev(t.cache.tables[0, p // 16].astype(np.int64) * 16 + p % 16)
        if value is not None:
            t.cache.k[slot] = value
            t.cache.v[slot] = value
        t.run()
        return t, ~left
    t, right = branches(bad)
    want, _ = branches(None)
    assert torch.equal(t.out[dev(right)], want.out[dev(right)]) and torch.isfinite(t.out[dev(right)]).all()
    if bad != bad:
        assert torch.isnan(t.out[dev(~right)]).all()                   # a row that sees them is not finite either


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_tables_with_entries_outside_the_cache(dtype):
    t = Tree(dtype, [200, 40], [9, 3], 1, 4, 2, 64, 16, seed=6)
    t.cache.tables[0, [2, 7, 13]] = [-1, 1 << 30, t.cache.k.shape[0] // 16]
    t.bt.copy_(dev(t.cache.tables))
    t.run()
    t.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_trees_in_a_padded_batch(dtype):
    t = Tree(dtype, [90, 3], [5, 2], 1, 16, 4, 64, 16, seed=11, first=70, behind=5000)
    t.run()
    got = to_f64(t.out)
    assert not got[:70].any() and not got[77:].any()
    t.off, t.mask, t.q, t.out = t.off - 70, t.mask[70: 77], t.q[70: 77], t.out[70: 77]
    t.check()


def test_tree_contexts_past_the_table_are_cut():
    t = Tree("f32", [50, 30], [4, 3], 1, 2, 1, 64, 16, seed=7)
    t.ctx[1] = 1 << 30
    t.cache.tables[1] = t.cache.tables[0]
    t.cache.k.nan_to_num_(0.5)
    t.cache.v.nan_to_num_(0.5)
    t.dev[1].copy_(dev(t.ctx))
    t.bt.copy_(dev(t.cache.tables))
    t.run()
    t.check()


# ---- selected blocks ------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hkv,d,bs", [(8, 128, 16), (1, 64, 5), (2, 64, 16), (3, 128, 1), (16, 128, 64), (5, 64, 33)])
@pytest.mark.parametrize("rows", [1, 60, 1300, 4600])
def test_block_bounds(dtype, hkv, d, bs, rows):
    rng = np.random.default_rng(rows + hkv + bs)
    n = rng.multinomial(rows, np.ones(min(rows, 7)) / min(rows, 7))
    begin = rng.integers(0, bs, len(n))
    c = Cache(rng, begin + n, DT[dtype], hkv, d, bs)
    slots = np.concatenate([c.tables[s, p // bs].astype(np.int64) * bs + p % bs for s, (b, m) in enumerate(zip(begin, n)) for p in [np.arange(b, b + m)]])
    slots[rng.random(rows) < 0.05] = -1
    slots[rng.random(rows) < 0.02] = c.k.shape[0]
    blocks = c.k.shape[0] // bs
    b0, s0 = rng.integers(-127, 128, (blocks, hkv, 2, d)).astype(np.int8), rng.random((blocks, hkv)).astype(np.float32)
    bounds, scales, slot = dev(b0), dev(s0), dev(slots)
    ab.alora_block_bounds(c.k, slot, bounds, scales, ab.make_bounds_dims(c.k, slot, hkv, d, bs))
    wb, ws = od.block_bounds(to_f64(c.k), slots, b0, s0, bs, hkv, d)
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(bounds.cpu().numpy(), wb)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_bounds_of_values_at_the_ends_of_their_range(dtype):
    bs, hkv, d = 4, 2, 64
    k = np.random.default_rng(1).standard_normal((9 * bs, hkv, d)).astype(np.float32)
    k[0, 0, 3], k[5, 1, 0], k[9, 0, 63], k[12:16], k[16:20] = np.nan, np.inf, -np.inf, 0.0, 1e-35
    k[20:24] *= 1e36
    k[24:28, 1] = -np.abs(k[24:28, 1])
    k[28, 0] = -0.0
    kt, slot = dev(k.reshape(-1, hkv * d)).to(DT[dtype]), dev(np.arange(36))
    bounds, scales = torch.ones((9, hkv, 2, d), dtype=torch.int8, device="cuda"), torch.ones((9, hkv), device="cuda")
    ab.alora_block_bounds(kt, slot, bounds, scales, ab.make_bounds_dims(kt, slot, hkv, d, bs))
    wb, ws = od.block_bounds(to_f64(kt), np.arange(36), np.zeros((9, hkv, 2, d), np.int8), np.zeros((9, hkv), np.float32), bs, hkv, d)
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(bounds.cpu().numpy(), wb)
    assert np.isinf(ws).sum() == 3 and not wb[3].any()


def test_bounds_in_a_padded_batch():
    """A block's next row may be thousands of rows without a slot further on, or not there."""
    bs, hkv, d = 16, 2, 64
    k = np.random.default_rng(2).standard_normal((6 * bs, hkv * d)).astype(np.float32)
    for gap, tail in ((1500, 0), (511, 4000), (512, 1), (513, 700), (0, 3000)):
        slots = np.concatenate([np.arange(40), np.full(gap, -1), np.arange(40, 75), np.full(tail, 96)])
        b0, s0 = np.ones((6, hkv, 2, d), np.int8), np.ones((6, hkv), np.float32)
        kt, slot, bounds, scales = dev(k), dev(slots), dev(b0), dev(s0)
        ab.alora_block_bounds(kt, slot, bounds, scales, ab.make_bounds_dims(kt, slot, hkv, d, bs))
        wb, ws = od.block_bounds(to_f64(kt), slots, b0, s0, bs, hkv, d)
        assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(bounds.cpu().numpy(), wb), (gap, tail)


class Select:
    """Random bounds over a pool; rows of several sequences."""

    def __init__(self, dtype, ctx, hq, hkv, d, bs, seed=0, coarse=False, spoiled=False):
        rng = self.rng = np.random.default_rng(seed)
        self.dt, self.sizes, self.bs = DT[dtype], (hq, hkv, d), bs
        self.cache = Cache(rng, np.array(ctx) + 1, self.dt, hkv, d, bs)
        blocks = self.cache.k.shape[0] // bs
        self.seq, self.pos = np.arange(len(ctx), dtype=np.int32), np.array(ctx, np.int32)
        top = 2 if coarse else 128
        self.bounds = rng.integers(-top + 1, top, (blocks, hkv, 2, d)).astype(np.int8)
        self.scales = (np.ones((blocks, hkv)) if coarse else rng.random((blocks, hkv))).astype(np.float32)
        self.q = values(rng, (len(ctx), hq * d), self.dt)
        if coarse:
            self.q.copy_(self.q.sign() * 0.5)
        if spoiled:
            self.scales[rng.random(self.scales.shape) < 0.05] = np.inf
            self.cache.tables[rng.random(self.cache.tables.shape) < 0.1] = 1 << 30
            self.seq[1], self.pos[2], self.seq[3] = -1, -7, len(ctx)
            self.pos[4] += 1 << 20                                     # (past the table: what its last block holds behind the sequence counts too)
            self.cache.k.nan_to_num_(0.3)
            self.cache.v.nan_to_num_(0.3)
        self.bt, self.dev = dev(self.cache.tables), [dev(self.seq), dev(self.pos)]
        self.b, self.s = dev(self.bounds), dev(self.scales)
        self.dims = ab.make_attn_dims(self.q, self.cache.k, self.bt, hq, hkv, d, bs)

    def select(self, budget, first, recent):
        hq, hkv, d = self.sizes
        self.selected = torch.full((len(self.seq), hkv, budget), -9, dtype=torch.int32, device="cuda")
        ws = torch.full((ab.alora_block_select_workspace_bytes(self.dims) + 16,), 255, dtype=torch.uint8, device="cuda")
        ab.alora_block_select(self.q, self.b, self.s, self.bt, *self.dev, self.selected, first, recent, self.dims, ws)
        want = od.block_select(to_f64(self.q), self.bounds, self.scales, self.cache.tables, self.seq, self.pos, self.bs, budget, first, recent, hq, hkv, d)
        got = self.selected.cpu().numpy()
        assert np.array_equal(got, want), (np.argwhere(got != want)[:5], got[got != want][:5], want[got != want][:5])

    def attend(self, lists=None):
        hq, hkv, d = self.sizes
        if lists is not None:
            self.selected = dev(lists)
        budget = self.selected.shape[-1]
        out = torch.full_like(self.q, float("nan"))
        ws = torch.full((ab.alora_selected_attention_workspace_bytes(self.dims, budget) // 4 + 4,), float("nan"), device="cuda")
        ab.alora_selected_attention(self.q, self.cache.k, self.cache.v, self.bt, *self.dev, self.selected, out, self.dims, ws)
        q, k, v, sel = to_f64(self.q), to_f64(self.cache.k), to_f64(self.cache.v), self.selected.cpu().numpy()
        close(out, q, k, v, d ** -0.5, hq, hkv, d, self.dt,
              lambda v: od.selected_attention(q, k, v, self.cache.tables, self.seq, self.pos, sel, self.bs, hq, hkv, d))
        return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("bs", [16, 5, 64])
def test_selection_and_attention(dtype, d, group, bs):
    t = Select(dtype, [0, 15, 16, 400, 777, 3000], 2 * group, 2, d, bs, seed=d + group)
    print("select", dtype, d, group, bs, flush=True)
    for budget, first, recent in ((1, 0, 1), (7, 1, 2), (40, 0, 3)):
        t.select(budget, first, recent)
        t.attend()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_scores_go_to_the_lower_block(dtype):
    t = Select(dtype, [4000, 999, 64, 17, 100, 5], 8, 2, 64, 4, seed=1, coarse=True)
    for budget, first, recent in ((2, 0, 1), (30, 2, 2), (64, 0, 1), (255, 0, 1), (256, 255, 1), (257, 0, 257), (1000, 1, 1), (1001, 1, 1)):
        t.select(budget, first, recent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_scales_and_tables_out_of_range(dtype):
    t = Select(dtype, [500, 20, 30, 40, 300, 700, 1], 4, 1, 128, 4, seed=2, spoiled=True)
    for budget, first, recent in ((3, 0, 1), (50, 4, 4), (170, 1, 1)):
        t.select(budget, first, recent)
        out = t.attend()
        assert not out[1:4].any()


def test_queries_that_are_zero_or_not_finite():
    t = Select("f32", [300] * 5, 4, 2, 64, 4, seed=3)
    t.q[0] = 0
    t.q[1, :256] = float("nan")
    t.q[2, 5] = float("inf")
    t.q[3] *= 1e-36
    t.q[4] *= 1e35
    hq, hkv, d = t.sizes
    selected = torch.empty((5, 2, 9), dtype=torch.int32, device="cuda")
    ws = torch.empty((ab.alora_block_select_workspace_bytes(t.dims) + 16,), dtype=torch.uint8, device="cuda")
    ab.alora_block_select(t.q, t.b, t.s, t.bt, *t.dev, selected, 1, 1, t.dims, ws)
    got = selected.cpu().numpy()
    flat = [*range(8), 75]                                             # all scores equal
    assert got[0].tolist() == [flat] * 2 and got[1].tolist() == [flat] * 2 and got[2, 0].tolist() == flat and got[3].tolist() == [flat] * 2
    rest = od.block_select(to_f64(t.q)[4:], t.bounds, t.scales, t.cache.tables, t.seq[4:], t.pos[4:], 4, 9, 1, 1, hq, hkv, d)
    assert np.array_equal(got[4:], rest)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_contexts(dtype):
    """More blocks than a workgroup's threads take at once, from one row to more than the chip holds at once."""
    for ctx, hkv, budget in (([70000], 1, 200), ([20000, 100, 9000], 8, 33), (list(range(3, 4000, 29)), 2, 20)):
        t = Select(dtype, ctx, 4 * hkv, hkv, 64, 8, seed=4)
        print("long", dtype, len(ctx), flush=True)
        t.select(budget, 1, 4)
        t.attend()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_one_sequence(dtype):
    """A chunk: 40 rows of two sequences, each with its own choice."""
    t = Select(dtype, [700, 90], 8, 2, 128, 16, seed=8)
    rng = np.random.default_rng(9)
    t.seq, t.pos = np.repeat([0, 1], 20).astype(np.int32), np.concatenate([np.arange(681, 701), np.arange(71, 91)]).astype(np.int32)
    t.q = values(rng, (40, 8 * 128), t.dt)
    t.dev, t.dims = [dev(t.seq), dev(t.pos)], ab.make_attn_dims(t.q, t.cache.k, t.bt, 8, 2, 128, 16)
    for budget in (4, 13):
        t.select(budget, 1, 2)
        t.attend()


@pytest.mark.parametrize("rows", [170, 300])
def test_more_lists_than_the_chip_holds(rows):
    """The longest contexts are looked through first; some rows are out of range."""
    rng = np.random.default_rng(rows)
    t = Select("bf16", rng.integers(0, 1500, rows), 8, 8, 64, 16, seed=10, spoiled=True)
    t.select(17, 1, 2)
    out = t.attend()
    assert not out[1:4].any()


@pytest.mark.parametrize("coarse", [False, True])
def test_more_blocks_than_threads_keep(coarse):
    """Blocks of one position: 40000 of them, and, in one kernel and in two, numbers of blocks around what a thread keeps."""
    t = Select("bf16", [40000, 200, 33000], 2, 1, 64, 1, seed=5, coarse=coarse)
    for budget, first, recent in ((300, 1, 2), (1, 0, 1), (33000, 5, 5)):
        t.select(budget, first, recent)
    for hkv, ctx in ((1, [1022, 1023, 1024, 1025, 2046, 2047, 2048, 2049, 8191, 8192]), (32, [767, 768, 1791, 1792, 1793, 2000, 4350, 4351])):
        t = Select("f32", ctx, hkv, hkv, 64, 1, seed=6, coarse=coarse)
        t.select(64, 1, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_of_any_kind(dtype):
    """Entries twice, out of order, outside the context, with holes, and none at all."""
    t = Select(dtype, [200, 200, 90, 31, 0], 8, 2, 128, 16, seed=5)
    lists = np.full((5, 2, 11), -1, np.int32)
    lists[0, 0] = [0, 0, 1, 1, 1, 5, 12, 12, 13, 99, 2 ** 31 - 1]
    lists[0, 1] = [12, 3, 4, 3, -1, 3, -5, 7, 7, 8, 2]
    lists[1] = [-1, -1, -1, -1, -1, -1, -1, -1, -1, -1, 12]
    lists[2, 0] = np.arange(11)
    lists[4, :, 0] = 0
    out = t.attend(lists)
    assert not out[3].any() and not out[2, 4 * 128:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_caches_and_bounds_past_4_gib(dtype):
    """The same blocks at the end of a pool whose byte offsets pass 32 bits (blocks of one position, so that those of the bounds do too): the same results, bit by bit."""
    hq, hkv, d = 16, 8, 128
    s = Select(dtype, [600, 90], hq, hkv, d, 1, seed=12)
    t = Tree(dtype, [500, 40], [20, 7], 1, hq, hkv, d, 1, seed=12)
    n = 2_200_000

    def moved(c):
        k = [torch.empty((n, hkv * d), dtype=s.dt, device="cuda") for _ in range(2)]
        for x, y in zip(k, (c.k, c.v)):
            x[-y.shape[0]:] = y
        return k, dev(np.where(c.tables >= 0, c.tables + n - c.k.shape[0], -1).astype(np.int32))

    def run(k, v, bt, bounds, scales, shift):
        slots = s.cache.tables[0, :601].astype(np.int64) + shift
        slot = dev(slots)
        ab.alora_block_bounds(k, slot, bounds, scales, ab.make_bounds_dims(k, slot, hkv, d, 1))
        dims, sel, out = ab.make_attn_dims(s.q, k, bt, hq, hkv, d, 1), torch.empty((2, hkv, 50), dtype=torch.int32, device="cuda"), torch.empty_like(s.q)
        ws = [torch.empty((m + 16,), dtype=torch.uint8, device="cuda") for m in (ab.alora_block_select_workspace_bytes(dims), ab.alora_selected_attention_workspace_bytes(dims, 50))]
        ab.alora_block_select(s.q, bounds, scales, bt, *s.dev, sel, 1, 2, dims, ws[0])
        ab.alora_selected_attention(s.q, k, v, bt, *s.dev, sel, out, dims, ws[1])
        return sel, out, bounds[slot], scales[slot]
    near = run(s.cache.k, s.cache.v, s.bt, s.b, s.s, 0)
    (k, v), bt = moved(s.cache)
    bounds, scales, m = torch.empty((n, hkv, 2, d), dtype=torch.int8, device="cuda"), torch.empty((n, hkv), device="cuda"), s.cache.k.shape[0]
    bounds[-m:], scales[-m:] = dev(s.bounds), dev(s.scales)
    far = run(k, v, bt, bounds, scales, n - m)
    assert all(torch.equal(x, y) for x, y in zip(near, far)) and torch.isfinite(near[1]).all()
    near = t.run().clone()
    (k, v), bt = moved(t.cache)
    ab.alora_tree_attention(t.q, k, v, bt, *t.dev, t.out, ab.make_attn_dims(t.q, k, bt, hq, hkv, d, 1), t.ws)
    assert torch.equal(t.out, near) and torch.isfinite(near).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seqs,columns", [(0, 4), (3, 0), (70, 0)])
def test_rows_without_sequences_or_tables(dtype, seqs, columns):
    """A batch padded to its size of which nothing is left, and sequences whose table has no room: zeros, no blocks."""
    dt, n = DT[dtype], 130
    q, kv = torch.ones((n, 512), device="cuda").to(dt), torch.full((32, 128), float("nan"), device="cuda").to(dt)
    bt = torch.zeros((seqs, columns), dtype=torch.int32, device="cuda")
    dims = ab.make_attn_dims(q, kv, bt, 8, 2, 64, 16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    off = i32(np.linspace(0, n if seqs else 0, seqs + 1).astype(int))
    ctx, mask, pos = i32([5] * seqs), torch.full((n, 1), -1, dtype=torch.int64, device="cuda"), i32([-9] * n)
    ws = torch.empty((ab.alora_tree_attention_workspace_bytes(dims, 1) + 16,), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, float("nan"))
    ab.alora_tree_attention(q, kv, kv, bt, off, ctx, mask, out, dims, ws)
    assert not out.any()
    ab.alora_tree_rows(i32([-1] * n), off, ctx, mask, pos)
    assert bool(mask.any()) == bool(seqs) and pos.tolist() == [5 if seqs else 0] * n
    seq, at = torch.arange(n, device="cuda").int() % max(1, seqs), i32([3] * n)
    b, s = torch.zeros((2, 2, 2, 64), dtype=torch.int8, device="cuda"), torch.zeros((2, 2), device="cuda")
    sel = torch.full((n, 2, 3), 7, dtype=torch.int32, device="cuda")
    ab.alora_block_select(q, b, s, bt, seq, at, sel, 1, 1, dims, None)
    assert (sel == -1).all()
    out.fill_(float("nan"))
    more = torch.empty((ab.alora_selected_attention_workspace_bytes(dims, 3) + 16,), dtype=torch.uint8, device="cuda")
    ab.alora_selected_attention(q, kv, kv, bt, seq, at, torch.zeros_like(sel), out, dims, more)
    assert not out.any()


def test_workspaces_that_are_not_dense_are_refused():
    t, s = Tree("f32", [50], [3], 1, 2, 1, 64, 16), Select("f32", [900], 2, 1, 64, 1)
    for bad in (torch.empty((1,), device="cuda").expand(1 << 28), torch.empty((1 << 23,), device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            ab.alora_tree_attention(t.q, t.cache.k, t.cache.v, t.bt, *t.dev, t.out, t.dims, bad)
        sel = torch.zeros((1, 1, 9), dtype=torch.int32, device="cuda")
        with pytest.raises(ValueError, match="workspace"):
            ab.alora_block_select(s.q, s.b, s.s, s.bt, *s.dev, sel, 1, 1, s.dims, bad)
        with pytest.raises(ValueError, match="workspace"):
            ab.alora_selected_attention(s.q, s.cache.k, s.cache.v, s.bt, *s.dev, sel, torch.empty_like(s.q), s.dims, bad)


# ---- streams, graphs ------------------------------------------------------------------------------
def test_another_stream_and_a_replayed_graph():
    """Tree and selection recorded once and replayed over changed data, with eager calls between the replays; two graphs, each with its workspace."""
    t, s = Tree("bf16", [900, 40], [30, 9], 1, 8, 2, 128, 16, seed=9), Select("bf16", [3000, 50, 700], 8, 2, 128, 16, seed=9)
    hq, hkv, d = s.sizes
    sel = torch.empty((3, 2, 12), dtype=torch.int32, device="cuda")
    ws = [torch.empty((max(16, n),), dtype=torch.uint8, device="cuda") for n in (ab.alora_block_select_workspace_bytes(s.dims), ab.alora_selected_attention_workspace_bytes(s.dims, 12))]
    out = torch.empty_like(s.q)
    slot = dev(np.arange(s.cache.k.shape[0]))
    dims = ab.make_bounds_dims(s.cache.k, slot, hkv, d, 16)
    s.cache.k.nan_to_num_(0.1)
    parents = dev(parents_of(t.rng, [30, 9]))
    pos = torch.empty((39,), dtype=torch.int32, device="cuda")
    step = step_case(np.random.default_rng(3), 40, 16, 9, 12, 2)

    def tree():
        ab.alora_tree_rows(parents, t.dev[0], t.dev[1], t.dev[2], pos)
        ab.alora_tree_attention(t.q, t.cache.k, t.cache.v, t.bt, *t.dev, t.out, t.dims, t.ws)

    def sparse():
        step.run()
        ab.alora_block_bounds(s.cache.k, slot, s.b, s.s, dims)
        ab.alora_block_select(s.q, s.b, s.s, s.bt, *s.dev, sel, 1, 2, s.dims, ws[0])
        ab.alora_selected_attention(s.q, s.cache.k, s.cache.v, s.bt, *s.dev, sel, out, s.dims, ws[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tree()
        sparse()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    step.check()
    graphs = []
    for work in (tree, sparse):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            work()
        graphs.append(g)
    for i in range(4):
        t.q.mul_(-0.9)
        s.q.mul_(-1.1)
        s.cache.k.mul_(0.95)
        for x in (t.out, out):
            x.fill_(float("nan"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in (t.out, sel, out, s.b)]
        tree()
        sparse()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (t.out, sel, out, s.b))), i
        step.check()
