"""What is timed of a decode step whose lengths are known on the GPU, of trees of drafted tokens, and of long contexts read in part.

Five kinds of work, calls of paper_2512_17910_amd.binding:

  steps      block tables, slots and rows of a step from the requests' lengths (alora_step_rows): requests grow, give drafts back or end;
             blocks come from and go back to a pool on the GPU.
  tree-rows  for every drafted token the bits of its ancestors and its position (alora_tree_rows).
  tree       attention of drafted tokens over the cache (alora_tree_attention): a row sees its sequence's context and its ancestors.
  bounds     bounds in 8 bits of the keys of the blocks that a step has written (alora_block_bounds).
  sparse     a layer of decoding over a few blocks of each context: those whose bounds promise the largest scores (alora_block_select) are
             read (alora_selected_attention).

Shapes are those of the repository's configurations (32 / 8 and 64 / 8 heads of 128, the small fp32 layer with 4 / 2 heads of 64, a server
of 256 requests) and generic ones in between.  Lengths, trees and the cases' other sizes follow from the case ("shape" is their seed); values and
the places of blocks in the pool follow from the seed.  Keys of a block lie around a vector of their own and queries near some blocks'
vectors, as texts that change their subject leave them.
"""
import math

import numpy as np
import torch

own = False             # the tools set it: run() calls the library's operators, not their plain forms

DEV = "cuda"
FLT_MAX = 3.4028234663852886e38
TINY = 2.0 ** -100      # bounds and queries below it count as zero


def listed():
    return [
        # a batch decodes one token each, some requests end or give drafts back.  The smallest call: launches and the host count
        {"name": "steps-decode-64", "kind": "steps", "seqs": 64, "mode": "decode", "most": 1, "max_blocks": 128, "bs": 16, "pad": 0, "short": False,
         "shape": 1},
        # prompts of many requests are admitted beside decoding ones: a large chunked prefill step
        {"name": "steps-prompts-90", "kind": "steps", "seqs": 90, "mode": "prompts", "most": 4000, "max_blocks": 1100, "bs": 16, "pad": 777, "short": False,
         "shape": 2},
        # a few requests with ordinary trees
        {"name": "tree-rows-16", "kind": "tree-rows", "seqs": 16, "nodes": 25, "words": 1, "shape": 3},
        # a busy server with wide trees
        {"name": "tree-rows-256", "kind": "tree-rows", "seqs": 256, "nodes": 200, "words": 4, "shape": 4},
        # one conversation with a small tree: few columns, a long axis
        {"name": "tree-1", "kind": "tree", "dtype": "bf16", "seqs": 1, "ctx": 9001, "nodes": 13, "words": 1, "hq": 32, "hkv": 8, "d": 128, "bs": 16,
         "shape": 5},
        # the small layer in reference precision, blocks of an odd size
        {"name": "tree-5-f32", "kind": "tree", "dtype": "f32", "seqs": 5, "ctx": 700, "nodes": 31, "words": 1, "hq": 4, "hkv": 2, "d": 64, "bs": 12,
         "shape": 6},
        # a batch of the large model with wide trees over ragged contexts
        {"name": "tree-48", "kind": "tree", "dtype": "bf16", "seqs": 48, "ctx": 16000, "nodes": 64, "words": 1, "hq": 64, "hkv": 8, "d": 128, "bs": 16,
         "shape": 7},
        # the keys that a decode step of 256 requests has written
        {"name": "bounds-decode-256", "kind": "bounds", "dtype": "bf16", "rows": 256, "seqs": 256, "hkv": 8, "d": 128, "bs": 16, "shape": 8},
        # those of a large prefill step
        {"name": "bounds-chunk-8192", "kind": "bounds", "dtype": "bf16", "rows": 8192, "seqs": 5, "hkv": 8, "d": 128, "bs": 16, "shape": 9},
        # one very long conversation
        {"name": "sparse-1", "kind": "sparse", "dtype": "bf16", "rows": 1, "seqs": 1, "ctx": 131000, "budget": 128, "first": 1, "recent": 4, "hq": 32,
         "hkv": 8, "d": 128, "bs": 16, "shape": 10},
        # the small layer in reference precision, a few rows of each sequence
        {"name": "sparse-7-f32", "kind": "sparse", "dtype": "f32", "rows": 7, "seqs": 3, "ctx": 2500, "budget": 24, "first": 1, "recent": 2, "hq": 4,
         "hkv": 2, "d": 64, "bs": 16, "shape": 11},
        # a busy server with long ragged contexts
        {"name": "sparse-200", "kind": "sparse", "dtype": "bf16", "rows": 200, "seqs": 200, "ctx": 24000, "budget": 100, "first": 1, "recent": 4, "hq": 32,
         "hkv": 8, "d": 128, "bs": 16, "shape": 12},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    u, shape = rng.random(), rng.randint(100, 1 << 30)
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    hkv, d, bs = rng.choice([1, 2, 4, 8, 8, 8]), rng.choice([64, 128, 128]), rng.choice([16, 16, 16, 32, 64, 8, 12, 5])
    hq = hkv * rng.choice([1, 2, 4, 4, 8])
    row = 2 * hkv * d * (2 if dtype == "bf16" else 4)                               # bytes of a position's keys and values
    if u < 0.2:
        mode = rng.choice(["decode", "drafts", "prompts"])
        seqs = _log_int(rng, 1, 90 if mode == "prompts" else 2000)
        most = {"decode": 1, "drafts": rng.randint(2, 64), "prompts": _log_int(rng, 16, 4000)}[mode]
        return {"kind": "steps", "seqs": seqs, "mode": mode, "most": most, "max_blocks": -(-most // bs) + rng.randint(8, 600), "bs": bs,
                "pad": rng.choice([0, rng.randint(1, 100)]), "short": rng.random() < 0.25, "shape": shape}
    if u < 0.35:
        words = rng.choice([1, 1, 2, 3, 4])
        return {"kind": "tree-rows", "seqs": _log_int(rng, 1, 256), "nodes": rng.randint(1, min(64 * words, 200)), "words": words, "shape": shape}
    if u < 0.6:
        words = rng.choice([1, 1, 1, 2, 4])
        nodes, ctx = _log_int(rng, 1, min(64 * words, 150)), _log_int(rng, 8, 16000)
        cost = ctx * max(row, 4 * hq * d * nodes // 400)                            # of a sequence, bytes or products at their rates
        seqs = max(1, min(_log_int(rng, 1, 48), 700_000_000 // cost))
        return {"kind": "tree", "dtype": dtype, "seqs": seqs, "ctx": ctx, "nodes": nodes, "words": words, "hq": hq, "hkv": hkv, "d": d, "bs": bs, "shape": shape}
    if u < 0.75:
        rows = _log_int(rng, 1, 8192)
        return {"kind": "bounds", "dtype": dtype, "rows": rows, "seqs": rows if rng.random() < 0.5 and rows <= 512 else min(rows, rng.randint(1, 9)), "hkv": hkv,
                "d": d, "bs": bs, "shape": shape}
    ctx = _log_int(rng, 16, 60000)
    rows = max(1, min(_log_int(rng, 1, 200), 5_000_000_000 // (ctx * row)))
    first, recent = rng.randint(0, 3), rng.randint(1, 6)
    return {"kind": "sparse", "dtype": dtype, "rows": rows, "seqs": rows if rng.random() < 0.7 else max(1, rows // rng.randint(2, 9)), "ctx": ctx,
            "budget": first + recent + _log_int(rng, 1, 90 * 16 // bs), "first": first, "recent": recent, "hq": hq, "hkv": hkv, "d": d, "bs": bs,
            "shape": shape}


# ---- what a program has in hand -----------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class _Values:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.dtype = dtype

    def __call__(self, shape, std=1.0):
        x = torch.empty(shape, dtype=self.dtype, device=DEV).normal_(generator=self.g)
        return x if std == 1.0 else x.mul_(std)


def _up(a, b):
    return -(-a // b)


def _tables(rng, lens, bs, max_blocks, spare):
    """(tables padded with -1, blocks of the pool): each sequence's blocks somewhere in the pool."""
    blocks = _up(lens, bs)
    n = int(blocks.sum()) + spare
    perm = rng.permutation(n).astype(np.int32)
    tables = np.full((len(lens), max_blocks), -1, np.int32)
    at = np.arange(max_blocks)[None, :] < blocks[:, None]
    tables[at] = perm[: int(blocks.sum())]
    return tables, n


def _step_sizes(case):
    """(lengths, changes, kept blocks) of the requests, from the case alone."""
    rng = np.random.default_rng(case["shape"])
    s, bs, most = case["seqs"], case["bs"], case["most"]
    longest = case["max_blocks"] * bs - most
    n = rng.integers(1, longest + 1, s)
    if case["mode"] == "prompts":                       # prompts behind a cached prefix or none, the others decode
        new = rng.random(s) < 0.8
        n = np.where(new, rng.integers(0, max(1, longest // bs // 4) + 1, s) * (rng.random(s) < 0.5) * bs, n)
        c = np.where(new, rng.integers(most // 2, most + 1, s), 1)
    else:
        c = rng.integers(1, most + 1, s)
        back = rng.random(s) < 0.1                      # drafts given back, or the request's end
        c = np.where(back, np.where(rng.random(s) < 0.3, -n, -np.minimum(n, rng.integers(1, 65, s))), c)
    kept = n // bs // 2 * (rng.random(s) < 0.3)
    return n.astype(np.int32), c.astype(np.int32), kept.astype(np.int32)


class _Steps:
    def __init__(self, case, seed):
        rng, bs = np.random.default_rng(seed), case["bs"]
        n, c, kept = _step_sizes(case)
        need = int(np.maximum(_up(n + c, bs) - _up(n, bs), 0).sum())
        free = max(0, need - 1 - need // 5) if case["short"] else need + 40
        tables, blocks = _tables(rng, n, bs, case["max_blocks"], free)
        used = np.zeros(blocks, bool)
        used[tables[tables >= 0]] = True
        ring, first = np.full(blocks, -1, np.int32), int(rng.integers(0, blocks))
        ring[(first + np.arange(free)) % blocks] = rng.permutation(np.flatnonzero(~used)).astype(np.int32)
        self.n_slots, self.rows = blocks * bs, int(np.maximum(c, 0).sum()) + case["pad"]
        self.lengths, self.change, self.kept = _dev(n), _dev(c), _dev(kept)
        self.adapters = _dev(rng.integers(-1, 32, case["seqs"]).astype(np.int32))
        self.tables, self.pool = _dev(tables), _dev(ring)
        self.state = _dev(np.array([first, free, 0, 0, 0, 0], np.int32))
        new = lambda k, t=torch.int32: torch.empty((k,), dtype=t, device=DEV)
        self.lengths_out, self.state_out, self.offsets = new(case["seqs"]), new(6), new(case["seqs"] + 1)
        self.seq, self.pos, self.aid, self.slot = new(self.rows), new(self.rows), new(self.rows), new(self.rows, torch.int64)
        self.dims = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                self.dims = ab.make_step_dims(self.tables, case["bs"], self.rows, self.pool, self.n_slots)
            ab.alora_step_rows(self.lengths, self.change, self.kept, self.adapters, self.tables, self.pool, self.state, self.lengths_out, self.state_out,
                               self.offsets, self.seq, self.pos, self.aid, self.slot, self.dims)
            return self.tables, self.pool, self.lengths_out, self.state_out, self.offsets, self.seq, self.pos, self.aid, self.slot
        return _plain_steps(self, case)


def _trees(case):
    """(rows of each sequence, parent of every row inside its tree), from the case alone."""
    rng = np.random.default_rng(case["shape"])
    n = rng.integers(max(1, case["nodes"] // 4), case["nodes"] + 1, case["seqs"]) if case["seqs"] > 1 else np.array([case["nodes"]])
    if case["seqs"] > 8:
        n[rng.integers(0, case["seqs"])] = 0            # a request that drafts nothing
    at = np.concatenate([np.arange(m) for m in n]) if n.sum() else np.zeros(0, np.int64)
    near = rng.random(len(at)) < 0.5                    # half of the drafts follow the last one, the others branch off anywhere
    parents = np.where(near, at - 1, np.floor(rng.random(len(at)) * (at + 1)).astype(np.int64) - 1)
    return n.astype(np.int64), parents.astype(np.int32)


def _offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _contexts(case, most):
    rng = np.random.default_rng(case["shape"] + 1)
    s = case["seqs"]
    return np.array([most]) if s == 1 else np.exp(rng.uniform(math.log(max(1, most / 16)), math.log(most + 1), s)).astype(np.int64).clip(0, most)


class _TreeRows:
    def __init__(self, case, seed):
        n, parents = _trees(case)
        rng = np.random.default_rng(seed)
        self.parents, self.offsets = _dev(parents), _dev(_offsets(n))
        self.ctx = _dev(rng.integers(0, 16000, case["seqs"]).astype(np.int32))
        self.mask = torch.empty((len(parents), case["words"]), dtype=torch.int64, device=DEV)
        self.pos = torch.empty((len(parents),), dtype=torch.int32, device=DEV)

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            ab.alora_tree_rows(self.parents, self.offsets, self.ctx, self.mask, self.pos)
            return self.mask, self.pos
        seen = _plain_ancestors(self.parents, self.offsets, case)
        seq, at = _plain_places(self.offsets, self.parents.shape[0])
        row = seen[seq, at]
        depth = row.sum(-1) - 1
        bits = torch.nn.functional.pad(row, (0, 64 * case["words"] - row.shape[-1])).view(-1, case["words"], 64).long()
        self.mask.copy_((bits << torch.arange(64, device=DEV)).sum(-1))
        self.pos.copy_(self.ctx[seq] + depth)
        return self.mask, self.pos


class _Tree:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        n, parents = _trees(case)
        ctx = _contexts(case, case["ctx"])
        tables, blocks = _tables(rng, ctx + n, case["bs"], _up(case["ctx"] + case["nodes"], case["bs"]), 3)
        at, bits = np.arange(len(parents)) - np.repeat(_offsets(n)[:-1], n), np.zeros((len(parents), case["words"]), np.uint64)
        first = _offsets(n)
        seq = np.repeat(np.arange(len(n)), n)
        for t in range(len(parents)):                   # a parent's row is in front of its children's
            if parents[t] >= 0:
                bits[t] = bits[first[seq[t]] + parents[t]]
            bits[t, at[t] // 64] |= np.uint64(1) << np.uint64(at[t] % 64)
        self.n, self.ctx_host = n, ctx
        self.offsets, self.ctx, self.tables = _dev(first), _dev(ctx.astype(np.int32)), _dev(tables)
        self.mask = _dev(bits.view(np.int64))
        self.kc, self.vc = (values((blocks * case["bs"], case["hkv"] * case["d"])) for _ in range(2))
        self.q = values((len(parents), case["hq"] * case["d"]))
        self.out = torch.empty_like(self.q)
        self.dims = self.ws = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                self.dims = ab.make_attn_dims(self.q, self.kc, self.tables, case["hq"], case["hkv"], case["d"], case["bs"])
                self.ws = torch.empty(max(16, ab.alora_tree_attention_workspace_bytes(self.dims, case["words"])), dtype=torch.uint8, device=DEV)
            ab.alora_tree_attention(self.q, self.kc, self.vc, self.tables, self.offsets, self.ctx, self.mask, self.out, self.dims, self.ws)
            return self.out
        return _plain_tree(self, case)


class _Bounds:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        t, s, bs, hkv, d = case["rows"], case["seqs"], case["bs"], case["hkv"], case["d"]
        shape = np.random.default_rng(case["shape"])
        n = np.full(s, 1) if s == t else np.diff(np.concatenate([[0], np.sort(shape.choice(np.arange(1, t), s - 1, replace=False)), [t]])) if s > 1 else np.array([t])
        begin = shape.integers(0, 4096, s)
        tables, blocks = _tables(rng, begin % bs + n, bs, _up(bs + int(n.max()), bs), 2)
        seq = np.repeat(np.arange(s), n)
        p = np.concatenate([np.arange(b % bs, b % bs + m) for b, m in zip(begin, n)])
        self.slot = _dev(tables[seq, p // bs].astype(np.int64) * bs + p % bs)
        self.kc = _keys(values, blocks, case)
        self.bounds = torch.zeros((blocks, hkv, 2, d), dtype=torch.int8, device=DEV)
        self.scales = torch.zeros((blocks, hkv), device=DEV)
        self.dims = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                self.dims = ab.make_bounds_dims(self.kc, self.slot, case["hkv"], case["d"], case["bs"])
            ab.alora_block_bounds(self.kc, self.slot, self.bounds, self.scales, self.dims)
        else:
            _plain_bounds(self, case)
        return self.bounds * self.scales[:, :, None, None]          # the values that the 8 bits stand for


def _keys(values, blocks, case):
    """Keys of a pool: those of a block around a vector of its own."""
    width = case["hkv"] * case["d"]
    k = values((blocks, case["bs"], width))
    return k.add_(values((blocks, 1, width))).view(blocks * case["bs"], width)


class _Sparse:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        t, s, bs, hq, hkv, d = (case[k] for k in ("rows", "seqs", "bs", "hq", "hkv", "d"))
        seq, pos, lens = _sparse_rows(case)
        tables, blocks = _tables(rng, lens, bs, _up(case["ctx"] + t, bs), 2)
        self.seq, self.pos, self.tables = _dev(seq), _dev(pos), _dev(tables)
        self.kc, self.vc = _keys(values, blocks, case), values((blocks * bs, hkv * d))
        keys = self.kc.view(blocks, bs, hkv, d)
        self.bounds, self.scales = _quantized(keys.amin(1).float(), keys.amax(1).float())
        # a query near the keys of one of its blocks, each head with its own share of it
        some = tables[seq, (rng.random(t) * (pos // bs + 1)).astype(np.int64)]
        topic = keys[_dev(some.astype(np.int64)), 0]                                # [t, hkv, d]
        q = values((t, hkv, hq // hkv, d)) + topic[:, :, None, :] * values((t, hkv, hq // hkv, 1)).abs_()
        self.q = q.view(t, hq * d)
        self.out = torch.empty_like(self.q)
        self.selected = torch.empty((t, hkv, case["budget"]), dtype=torch.int32, device=DEV)
        self.dims = self.ws = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                self.dims = ab.make_attn_dims(self.q, self.kc, self.tables, case["hq"], case["hkv"], case["d"], case["bs"])
                self.ws = torch.empty(max(16, ab.alora_block_select_workspace_bytes(self.dims),
                                          ab.alora_selected_attention_workspace_bytes(self.dims, case["budget"])), dtype=torch.uint8, device=DEV)
            ab.alora_block_select(self.q, self.bounds, self.scales, self.tables, self.seq, self.pos, self.selected, case["first"], case["recent"], self.dims,
                                  self.ws)
            ab.alora_selected_attention(self.q, self.kc, self.vc, self.tables, self.seq, self.pos, self.selected, self.out, self.dims, self.ws)
            return self.selected, self.out
        return _plain_sparse(self, case)


def _sparse_rows(case):
    """(sequence and position of every row, lengths of the sequences), from the case alone: the last rows of each sequence."""
    t, s = case["rows"], case["seqs"]
    ctx = _contexts(case, case["ctx"])
    n = np.full(s, t // s)
    n[: t - int(n.sum())] += 1
    seq = np.repeat(np.arange(s), n)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(ctx, n)])
    return seq.astype(np.int32), pos.astype(np.int32), ctx + n


# ---- the plain forms ----------------------------------------------------------------------------
def _plain_steps(st, case):
    bs, cap, ring, blocks = case["bs"], case["max_blocks"] * case["bs"], st.pool.shape[0], st.n_slots // case["bs"]
    n, c, kept = st.lengths.long(), st.change.long(), st.kept.long()
    first, count = st.state[0].long(), st.state[1].long()
    valid = (n >= 0) & (n <= cap) & (n + c >= 0) & (n + c <= cap)
    have, want = (n + bs - 1) // bs, (n + c + bs - 1) // bs
    take = torch.where(valid, (want - have).clamp(min=0), 0)
    new = torch.where(valid, c.clamp(min=0), 0)
    take_upto, new_upto = take.cumsum(0), new.cumsum(0)
    ok = valid & ((c <= 0) | (take_upto <= count) & (new_upto <= st.rows))
    take, new = torch.where(ok, take, 0), torch.where(ok, new, 0)
    back = torch.where(ok, (have - torch.maximum(want, kept)).clamp(min=0), 0)
    take_at, new_at, back_at = take.cumsum(0) - take, new.cumsum(0), back.cumsum(0) - back
    st.lengths_out.copy_(torch.where(ok, n + c, n))
    st.offsets[0] = 0
    st.offsets[1:] = new_at
    # blocks go back: the last one first
    j = torch.arange(int(back.sum()), device=DEV)
    s = torch.searchsorted(back_at + back, j, right=True)
    st.pool[(first + count + j) % ring] = st.tables[s, have[s] - 1 - (j - back_at[s])]
    # blocks are taken
    k = torch.arange(int(take.sum()), device=DEV)
    s = torch.searchsorted(take_at + take, k, right=True)
    st.tables[s, have[s] + k - take_at[s]] = st.pool[(first + k) % ring]
    total = torch.stack((take.sum(), back.sum()))
    st.state_out.copy_(torch.stack(((first + total[0]) % ring, count - total[0] + total[1], new.sum(), total[0], total[1], (~ok).sum())))
    # rows
    r = torch.arange(st.rows, device=DEV)
    s = torch.searchsorted(new_at, r, right=True)
    live = s < case["seqs"]
    s = s.clamp(max=case["seqs"] - 1)
    p = torch.where(live, n[s] + r - (new_at - new)[s], 0)
    block = st.tables[s, p // bs].long()
    st.seq.copy_(torch.where(live, s, -1))
    st.pos.copy_(p)
    st.aid.copy_(torch.where(live, st.adapters[s], -1))
    st.slot.copy_(torch.where(live & (block >= 0) & (block < blocks), block * bs + p % bs, -1))
    return st.tables, st.pool, st.lengths_out, st.state_out, st.offsets, st.seq, st.pos, st.aid, st.slot


def _plain_places(offsets, rows):
    """Sequence and place in it of every row."""
    r = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(offsets[1:].long().contiguous(), r, right=True)
    return seq, r - offsets.long()[seq]


def _plain_ancestors(parents, offsets, case):
    """[sequences, nodes, nodes]: whether a node is another one's ancestor or itself, by squaring the steps to the parent."""
    seq, at = _plain_places(offsets, parents.shape[0])
    step = torch.zeros((case["seqs"], case["nodes"], case["nodes"]), device=DEV)
    step[seq, at, at] = 1.0
    has = parents >= 0
    step[seq[has], at[has], parents[has].long()] = 1.0
    for _ in range(max(1, (case["nodes"] - 1).bit_length())):
        step = (torch.bmm(step, step) > 0).float()
    return step > 0


def _plain_softmax(score, seen):
    """Weights of each row over what it sees; zeros where it sees nothing."""
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    return w / w.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_tree(st, case):
    s, hq, hkv, d, bs = (case[k] for k in ("seqs", "hq", "hkv", "d", "bs"))
    g, nodes, longest = hq // hkv, int(st.n.max()), int((st.ctx_host + st.n).max())
    ctx, n = st.ctx.long(), (st.offsets[1:] - st.offsets[:-1]).long()
    p = torch.arange(longest, device=DEV)
    slot = (st.tables[:, p // bs].long() * bs + p % bs).clamp(min=0)                # [s, longest]
    k, v = (x[slot].float().view(s, longest, hkv, d).transpose(1, 2) for x in (st.kc, st.vc))
    seq, at = _plain_places(st.offsets, st.q.shape[0])
    q = torch.zeros((s, nodes, hkv, g, d), device=DEV)
    q[seq, at] = st.q.float().view(-1, hkv, g, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(s * hkv, nodes * g, d)
    score = torch.bmm(q, k.reshape(s * hkv, longest, d).transpose(1, 2).contiguous()) / math.sqrt(d)
    bit = p[None, :] - ctx[:, None]                                                 # place in the tree of each position
    seen = torch.zeros((s, nodes, longest), dtype=torch.bool, device=DEV)
    word = (bit.clamp(min=0) // 64).clamp(max=case["words"] - 1)[seq]
    seen[seq, at] = (bit < 0)[seq] | ((bit < n[:, None])[seq] & ((st.mask.gather(1, word) >> (bit[seq].clamp(min=0) % 64)) & 1).bool())
    seen = seen[:, None, :, None, :].expand(s, hkv, nodes, g, longest).reshape(s * hkv, nodes * g, longest)
    out = torch.bmm(_plain_softmax(score, seen), v.reshape(s * hkv, longest, d))
    out = out.view(s, hkv, nodes, g, d).permute(0, 2, 1, 3, 4)[seq, at]
    st.out.copy_(out.reshape(-1, hq * d))
    return st.out


def _quantized(low, high):
    """Bounds in 8 bits, rounded outwards, and their scales; keys that are not finite give scale inf."""
    a = torch.maximum(low.abs(), high.abs()).amax(-1)
    full, fine = torch.full_like(a, 127.0), torch.isfinite(a)     # (a division by a number would be a product with its inverse)
    inv = torch.where(fine & (a >= TINY), full / a, 0.0)[..., None]
    q = lambda x, up: torch.nan_to_num((x * inv).ceil() if up else (x * inv).floor()).clamp(-127, 127).to(torch.int8)
    return torch.stack((q(high, True), q(low, False)), -2).contiguous(), torch.where(fine, a / full, math.inf)


def _plain_bounds(st, case):
    bs = case["bs"]
    block, off = st.slot // bs, st.slot % bs
    last = torch.ones_like(block, dtype=torch.bool)
    last[:-1] = block[1:] != block[:-1]
    block, off = block[last], off[last]
    k = st.kc.view(-1, bs, case["hkv"], case["d"])[block].float()
    past = (torch.arange(bs, device=DEV)[None, :] > off[:, None])[:, :, None, None]
    q, scale = _quantized(k.masked_fill(past, math.inf).amin(1), k.masked_fill(past, -math.inf).amax(1))
    st.bounds[block] = q
    st.scales[block] = scale


def _plain_sparse(st, case):
    t, hq, hkv, d, bs, budget = (case[k] for k in ("rows", "hq", "hkv", "d", "bs", "budget"))
    g, seq, pos = hq // hkv, st.seq.long(), st.pos.long()
    blocks = st.tables.shape[1]
    table = st.tables[seq].long()                                                   # [t, blocks]
    q = st.q.double().view(t, hkv, g, d)
    both = torch.cat((q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)), -1).float()    # [t, hkv, 2 d]
    a = both.abs().amax(-1, keepdim=True)
    both = torch.round(both * torch.where(a >= TINY, torch.full_like(a, 127.0) / a, 0.0))
    # whole numbers below 2^24: exact in every order of summation
    sums = torch.matmul(st.bounds.view(-1, hkv, 2 * d)[table.clamp(min=0)].permute(0, 2, 1, 3).float(), both[..., None])[..., 0]      # [t, hkv, blocks]
    scale = st.scales[table.clamp(min=0)].transpose(1, 2)
    score = torch.where(torch.isinf(scale), FLT_MAX, (sums * scale).clamp(-FLT_MAX, FLT_MAX))
    b, n = torch.arange(blocks, device=DEV), pos // bs + 1
    always = (b[None, :] < torch.minimum(n, n.new_tensor(case["first"]))[:, None]) | ((b[None, :] >= (n - case["recent"])[:, None]) & (b[None, :] < n[:, None]))
    score = torch.where(always[:, None, :], math.inf, score)
    score = torch.where((b[None, :] < n[:, None])[:, None, :], score, -math.inf)
    by_score = torch.sort(score, dim=-1, descending=True, stable=True).indices      # (ties: the lowest block first)
    best = by_score[..., :budget]
    best = torch.where(best < n[:, None, None], best, blocks).sort(-1).values
    best = torch.nn.functional.pad(best, (0, max(0, budget - blocks)), value=blocks)
    st.selected.copy_(torch.where(best < blocks, best, -1))
    # attention over the positions of the selected blocks
    at = torch.where(best < blocks, best, 0).contiguous()
    block = table.gather(1, at.view(t, -1)).view(t, hkv, budget)
    off = torch.arange(bs, device=DEV)
    slot = (block.clamp(min=0)[..., None] * bs + off).view(t, hkv, budget * bs)
    seen = ((best < blocks) & (block >= 0))[..., None] & (at[..., None] * bs + off <= pos[:, None, None, None])
    head = torch.arange(hkv, device=DEV)[None, :, None]
    k, v = (x.view(-1, hkv, d)[slot, head].float().view(t * hkv, budget * bs, d) for x in (st.kc, st.vc))
    score = torch.bmm(st.q.float().view(t * hkv, g, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
    w = _plain_softmax(score, seen.reshape(t * hkv, 1, budget * bs).expand(-1, g, -1))
    st.out.copy_(torch.bmm(w, v).view(t, hq * d))
    return st.selected, st.out


# ---- the definitions in 64 bits -----------------------------------------------------------------
def _exact_attention(q, k, v, seen):
    """q [columns, d], k and v [positions, d], seen [columns or 1, positions]"""
    x = (q @ k.T) * q.shape[-1] ** -0.5
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    x = torch.softmax(x, -1)
    return torch.nan_to_num(x) @ v


def exact(case, seed):
    if case["kind"] in ("steps", "tree-rows"):
        return None                                     # whole numbers
    if case["kind"] == "bounds":
        st = _Bounds(case, seed)
        bs, out = case["bs"], torch.zeros(st.bounds.shape, dtype=torch.float64, device=DEV)
        slots = st.slot.cpu().numpy()
        lasts = [int(x) for x, y in zip(slots, np.append(slots[1:], -1)) if y // bs != x // bs]
        keys = st.kc.view(-1, bs, case["hkv"], case["d"])
        for slot in lasts:                              # (the factor and its product are fp32 numbers by definition, as whole numbers follow from them)
            k = keys[slot // bs, : slot % bs + 1].double().cpu().numpy()
            for row, end, rounded in ((0, k.max(0), np.ceil), (1, k.min(0), np.floor)):
                a = np.abs(k).max((0, 2))[:, None]
                whole = rounded(end.astype(np.float32) * (np.float32(127) / a.astype(np.float32))).clip(-127, 127)
                out[slot // bs, :, row] = _dev(whole.astype(np.float64) * (a / 127.0))
        return out
    hq, hkv, d, bs = (case[k] for k in ("hq", "hkv", "d", "bs"))
    g = hq // hkv
    if case["kind"] == "tree":
        st = _Tree(case, seed)
        out = torch.zeros(st.q.shape, dtype=torch.float64, device=DEV)
        first = _offsets(st.n)
        bits = st.mask.cpu().numpy().view(np.uint64)
        for s in range(case["seqs"]):
            a, b, c = int(first[s]), int(first[s + 1]), int(st.ctx_host[s])
            if a == b:
                continue
            p = torch.arange(c + b - a, device=DEV)
            slot = st.tables[s, p // bs].long() * bs + p % bs
            j = np.arange(b - a)
            tree = (bits[a:b, j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1)
            seen = torch.cat((torch.ones((b - a, c), dtype=torch.bool, device=DEV), _dev(tree.astype(bool))), 1).repeat_interleave(g, 0)
            k, v = (x[slot].double().view(-1, hkv, d) for x in (st.kc, st.vc))
            q = st.q[a:b].double().view(b - a, hkv, g, d)
            got = [_exact_attention(q[:, h].reshape(-1, d), k[:, h], v[:, h], seen).view(b - a, g, d) for h in range(hkv)]
            out[a:b] = torch.stack(got, 1).reshape(b - a, hq * d)
        return out
    st = _Sparse(case, seed)
    out = torch.zeros(st.q.shape, dtype=torch.float64, device=DEV)
    seq, pos, _ = _sparse_rows(case)
    f32 = np.float32
    for t in range(case["rows"]):
        n = int(pos[t]) // bs + 1
        table = st.tables[int(seq[t]), :n].long()
        q = st.q[t].double().view(hkv, g, d)
        for h in range(hkv):
            x = q[h].cpu().numpy()
            both = np.concatenate([np.maximum(x, 0).sum(0), np.minimum(x, 0).sum(0)]).astype(f32)
            a = np.abs(both).max()
            both = np.rint(both * (f32(127) / a if a >= TINY else f32(0))).astype(np.float64)
            sums = (st.bounds[table, h].view(n, 2 * d).double() @ _dev(both)).cpu().numpy()
            score = sums.astype(f32) * st.scales[table, h].cpu().numpy()
            rest = [b for b in np.argsort(-score, kind="stable") if case["first"] <= b < n - case["recent"]]
            always = [b for b in range(n) if b < case["first"] or b >= n - case["recent"]]
            chosen = np.sort(np.array(always + rest[: max(0, case["budget"] - len(always))]))
            p = (chosen[:, None] * bs + np.arange(bs)).reshape(-1)
            p = _dev(p[p <= pos[t]])
            slot = table[p // bs] * bs + p % bs
            k, v = (c[slot].double().view(-1, hkv, d)[:, h] for c in (st.kc, st.vc))
            out[t].view(hkv, g, d)[h] = _exact_attention(q[h], k, v, torch.ones((1, len(p)), dtype=torch.bool, device=DEV))
    return None, out


_KINDS = {"steps": _Steps, "tree-rows": _TreeRows, "tree": _Tree, "bounds": _Bounds, "sparse": _Sparse}


def prepare(case, seed):
    return case, _KINDS[case["kind"]](case, seed)


def run(state):
    case, st = state
    return st.run(case)


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    if case["kind"] == "steps":
        n, c, kept = _step_sizes(case)
        blocks = np.abs(_up(n + c, case["bs"]) - _up(n, case["bs"])).sum()          # moved between tables and pool
        return {"bytes": float(20 * (np.maximum(c, 0).sum() + case["pad"]) + 24 * case["seqs"] + 8 * blocks), "flops": 0.0}
    if case["kind"] == "tree-rows":
        n, _ = _trees(case)
        return {"bytes": float((8 + 8 * case["words"]) * n.sum() + 8 * case["seqs"]), "flops": 0.0}
    hkv, d, bs = (case[k] for k in ("hkv", "d", "bs"))
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "bounds":                        # about: where a sequence's rows begin inside a block is the case's
        blocks = case["rows"] if case["seqs"] == case["rows"] else case["rows"] / bs + case["seqs"]
        rows = blocks * (bs + 1) / 2 if case["seqs"] == case["rows"] else case["rows"] + case["seqs"] * bs / 2
        return {"bytes": rows * hkv * d * e + blocks * hkv * (2 * d + 4) + 8.0 * case["rows"], "flops": 2.0 * rows * hkv * d}
    hq = case["hq"]
    if case["kind"] == "tree":
        n, _ = _trees(case)
        seen = _contexts(case, case["ctx"]) + n
        return {"bytes": float(2 * seen.sum() * hkv * d * e + 2 * n.sum() * hq * d * e + 8 * case["words"] * n.sum()),
                "flops": float(4 * (n * seen).sum() * hq * d)}
    _, pos, _ = _sparse_rows(case)
    n = pos // bs + 1
    read = np.minimum(n, case["budget"])
    positions = (read - 1) * bs + pos % bs + 1
    scored = np.maximum(n - case["first"] - case["recent"], 0) * (n > case["budget"])  # blocks whose bounds have to be looked at
    return {"bytes": float(2 * positions.sum() * hkv * d * e + scored.sum() * hkv * (2 * d + 4) + 2 * len(pos) * hq * d * e + 4 * (scored + read).sum() * hkv),
            "flops": float(4 * positions.sum() * hq * d + 4 * scored.sum() * hkv * d)}
