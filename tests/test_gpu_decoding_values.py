"""Trees and selected blocks: how far weights are kept, and values that are not finite (alora_tree.h, alora_select.h).

Tolerances, per element, are those of test_gpu_decoding.py without its term for weights rounded to bf16 (2^-8 of A = sum_j w_j |v_j|): both readers take a
weight into the product with V as two bf16 numbers, the first cut off (its remainder is below 2^-7 of the weight), the second the remainder of the weight times
1 + 2^-9, rounded (half a step: 2^-8 of at most 2^-7 + 2^-9): 1.25 * 2^-15 of A.  The factor is every weight's, and the sum's they are divided by."""
import numpy as np
import pytest
import torch

from oracle import decoding as od
from paper_2512_17910_amd import binding as ab
from gpu_util import to_f64
from test_gpu_decoding import HALF, U32, Select, Tree, dev

pytestmark = pytest.mark.gpu

TWO_NUMBERS = {torch.bfloat16: 1.25 * 2.0 ** -15, torch.float32: 0.0}


def whole(got, q, k, v, hq, hkv, d, dt, attention):
    """attention(v): the oracle's rows for these values."""
    got, want, size = to_f64(got), attention(v), attention(np.abs(v))
    assert np.isfinite(got).all()
    kmax = np.nan_to_num(np.abs(k), nan=0.0).max(0).reshape(hkv, d)
    S = d ** -0.5 * (np.abs(q).reshape(-1, hkv, hq // hkv, d) * kmax[None, :, None]).sum(-1).reshape(-1, hq, 1)
    err = (((2 * d * S + 64) * U32 + TWO_NUMBERS[dt]) * size.reshape(-1, hq, d)).reshape(size.shape)
    over = np.abs(got - want) - (HALF[dt] * (np.abs(want) + err) + err)
    assert np.all(over <= 0), (float(over.max()), np.unravel_index(int(np.argmax(over)), over.shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 8])
@pytest.mark.parametrize("ctx,n", [([0, 33, 270, 1, 95, 600], [7, 1, 40, 0, 64, 3]), ([5000, 20], [13, 2])], ids=["ragged", "parts"])
def test_weights_of_trees(dtype, d, group, ctx, n):
    t = Tree(dtype, ctx, n, 1, 2 * group, 2, d, 16, seed=d + group)
    t.run()
    q, k, v = to_f64(t.q), to_f64(t.cache.k), to_f64(t.cache.v)
    whole(t.out, q, k, v, 2 * group, 2, d, t.dt, lambda v: od.tree_attention(q, k, v, t.cache.tables, t.off, t.ctx, t.mask, 16, 2 * group, 2, d))


def every_block(t, budget):
    """Lists of all blocks of the rows' contexts."""
    lists = np.full((len(t.pos), t.sizes[1], budget), -1, np.int32)
    for r, p in enumerate(t.pos):
        lists[r, :, : p // t.bs + 1] = np.arange(p // t.bs + 1)
    return lists


def attend(t, lists):
    out, sel = torch.full_like(t.q, float("nan")), dev(lists)
    ws = torch.full((ab.alora_selected_attention_workspace_bytes(t.dims, lists.shape[-1]) // 4 + 4,), float("nan"), device="cuda")
    ab.alora_selected_attention(t.q, t.cache.k, t.cache.v, t.bt, *t.dev, sel, out, t.dims, ws)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 8])
def test_weights_of_selected_blocks(dtype, d, group):
    t = Select(dtype, [0, 15, 16, 400, 777, 3000], 2 * group, 2, d, 16, seed=d + group)
    lists = every_block(t, 190)
    out = attend(t, lists)
    q, k, v = to_f64(t.q), to_f64(t.cache.k), to_f64(t.cache.v)
    whole(out, q, k, v, 2 * group, 2, d, t.dt, lambda v: od.selected_attention(q, k, v, t.cache.tables, t.seq, t.pos, lists, 16, 2 * group, 2, d))


INF, NAN = float("inf"), float("nan")


def slot_of(cache, seq, place, bs=16):
    return int(cache.tables[seq, place // bs]) * bs + place % bs


def spoilt(run, v, places, hq, hkv, d, sees):
    """run() with zeros and then with values that are not finite at places (sequence, slot, K/V head, component, value): what a row sees
    (sees(row, slot)) makes that component of its heads what the sum of such values is; everything else stays bit by bit."""
    for _, slot, g, c, _ in places:
        v[slot, g * d + c] = 0.0
    clean = run().clone()
    for _, slot, g, c, z in places:
        v[slot, g * d + c] = z
    got = run().clone()
    want = np.zeros((clean.shape[0], hq, d))
    with np.errstate(invalid="ignore"):
        for _, slot, g, c, z in places:
            for r in range(clean.shape[0]):
                if sees(r, slot):
                    want[r, g * (hq // hkv): (g + 1) * (hq // hkv), c] += z
    got, want, clean = to_f64(got), want.reshape(clean.shape), to_f64(clean)
    assert np.isfinite(clean).all() and not np.isfinite(want).all()
    wrong = np.where(np.isfinite(want), got != clean, ~((got == want) | (np.isnan(got) & np.isnan(want))))
    assert not wrong.any(), [(tuple(i), got[tuple(i)], want[tuple(i)]) for i in np.argwhere(wrong)[:6]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 8])
@pytest.mark.parametrize("all_blocks", [False, True])
def test_values_of_selected_blocks_that_are_not_finite(dtype, d, group, all_blocks):
    """One place alone (its weight is 1), some of many, two of different signs, and blocks that are not read."""
    hq = 2 * group
    t = Select(dtype, [0, 15, 400, 777, 3000], hq, 2, d, 16, seed=3 * d + group)
    lists = every_block(t, 190) if all_blocks else np.full((5, 2, 4), -1, np.int32)
    if not all_blocks:
        lists[:2, :, 0] = 0
        lists[2:, :, :3] = [[[0, 7, 25]], [[3, 8, 48]], [[5, 90, 187]]]
    at = [(0, 0, 1, 5, INF), (0, 0, 0, d - 1, -INF), (0, 0, 0, 0, NAN), (1, 3, 0, 7, INF), (1, 15, 0, 8, -INF), (2, 115, 1, 33, -INF), (2, 118, 1, 33, INF), (2, 5, 0, 0, INF),
          (2, 399, 0, 0, INF), (3, 60, 1, 17, -INF), (3, 63, 1, 18, NAN), (3, 130, 0, 62, INF), (4, 95, 0, 1, INF), (4, 1450, 0, 2, -INF), (4, 3000, 1, 40, INF), (4, 2000, 1, 41, INF)]
    of_row = {slot_of(t.cache, s, p): (s, p // 16) for s, p, *_ in at}
    spoilt(lambda: attend(t, lists), t.cache.v, [(s, slot_of(t.cache, s, p), g, c, z) for s, p, g, c, z in at], hq, 2, d,
           lambda r, slot: of_row[slot][0] == r and of_row[slot][1] in lists[r, 0].tolist())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", [0.0, -7.0, -30.0, -69.0, -87.0])
def test_infinite_values_of_small_weight(dtype, score):
    """One place of 300 with a score far below the others': its weight is a number of fp32 (2^-126 at least; the rest of it in bf16 has fewer bits), and an infinity of it is one."""
    d = 128
    t = Select(dtype, [299], 2, 2, d, 16, seed=4)
    t.q.fill_(1.0)
    t.cache.k.zero_()
    slot = slot_of(t.cache, 0, 133)
    t.cache.k[slot] = score / d ** 0.5
    lists = every_block(t, 20)
    spoilt(lambda: attend(t, lists), t.cache.v, [(0, slot, 0, 9, INF), (0, slot, 1, 100, -INF)], 2, 2, d, lambda r, s: True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [2, 8, 16])                             # (with two, wavefronts share the columns of the narrow trees)
def test_values_of_trees_that_are_not_finite(dtype, d, hq):
    """In drafts that some rows see, in the context's places beside them, and further forward; keys are finite."""
    ctx, n = [70, 9000, 31, 0], [41, 13, 64, 3]
    for few in (False, True):
        t = Tree(dtype, ctx[:2] if few else ctx, n[:2] if few else n, 1, hq, 2, d, 16, seed=hq + d)
        t.run()
        t.check()
        at = [(0, 70, 0, 3, INF), (0, 75, 1, 60, -INF), (0, 80, 1, 60, INF), (0, 97, 0, 33, NAN), (0, 110, 0, 34, INF), (0, 66, 1, 8, -INF), (0, 12, 1, 9, INF), (1, 9001, 0, 0, INF), (1, 9012, 0, 0, -INF),
              (1, 9005, 1, 17, NAN), (1, 9010, 1, 31, -INF), (1, 4321, 1, 32, INF), (1, 8999, 0, 47, INF)]
        if not few:
            at += [(2, 31, 0, 5, INF), (2, 40, 1, 6, INF), (2, 63, 1, 24, -INF), (2, 64, 1, 25, NAN), (2, 94, 0, 26, INF), (2, 30, 0, 13, -INF), (3, 0, 1, 14, INF), (3, 2, 0, 15, NAN)]
        places = {slot_of(t.cache, s, p): (s, p - ctx[s]) for s, p, *_ in at}

        def sees(r, slot):
            s, j = places[slot]
            return t.off[s] <= r < t.off[s + 1] and (j < 0 or bool(int(t.mask[r, 0]) >> j & 1))
        spoilt(t.run, t.cache.v, [(s, slot_of(t.cache, s, p), g, c, z) for s, p, g, c, z in at], hq, 2, d, sees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq", [2, 16])
@pytest.mark.parametrize("place", [10, 68, 70, 75])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_values_of_no_weight_that_are_not_finite(dtype, hq, place, bad):
    """A place that is seen counts however small its weight (e^-339, which fp32 does not know): the component is not finite, wherever the place lies -- far in front of
    the drafts, beside them, among them.  Rows that do not see it are as if it were not there."""
    d, ctx = 128, 70
    t = Tree(dtype, [ctx], [20], 1, hq, 2, d, 16, seed=6)
    t.q.fill_(1.0)
    t.cache.k.zero_()
    slot = slot_of(t.cache, 0, place)
    t.cache.k[slot] = -30.0
    t.cache.v[slot, 40] = 0.0
    want = to_f64(t.run()).reshape(20, hq, d)
    t.cache.v[slot, 40] = bad
    got = to_f64(t.run()).reshape(20, hq, d)
    seen = np.array([place < ctx or bool(int(m) >> (place - ctx) & 1) for m in t.mask[:, 0]])
    assert not np.isfinite(got[seen][:, : hq // 2, 40]).any() and (bad == bad or np.isnan(got[seen][:, : hq // 2, 40]).all())
    got[seen, : hq // 2, 40] = want[seen, : hq // 2, 40]
    assert np.array_equal(got, want)
    assert seen.any() and (place < 75 or not seen.all())
