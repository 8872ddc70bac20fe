#!/usr/bin/env python3
"""Conversations answered with drafted trees, and over a few blocks of their contexts: what alora_steps.h, alora_tree.h and alora_select.h are for, next to the
planner, the projection, the heads and the cache's moves.

  1. prompts are read, one conversation under an adapter, and answered token by token (planner, projection, heads, reader): the text to compare with;
  2. the same answers with trees of drafts.  Lengths, block tables and the pool of free blocks are on the device from here on.  A step gives every
     conversation rows for its tree (alora_step_rows), masks and positions (alora_tree_rows), goes through the layers (alora_tree_attention), takes the longest
     path that the model itself would have chosen, moves the path's rows together (alora_cache_move_rows, through spare slots) and gives the other places
     and their blocks back (alora_step_rows).  Nothing of it waits for the host;
  3. tokens are added over selected blocks: bounds of the blocks that a step writes (alora_block_bounds), a choice for every row and K/V head
     (alora_block_select), attention over it (alora_selected_attention); with a budget for all blocks, and with one for some.

Synthetic data.  Checks itself (the text of 2 is what a from-scratch computation of it would choose, its cache what 1 left; 3 with all blocks gives 1's rows) and
prints one JSON line.

    python -m paper_2512_17910_amd.speculation [--layers 4] [--prompt 1000] [--dtype bf16|f32] [--answer 40]
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from .conversation import NEVER, Model, _off

# A tree of eight drafts: the token that is known, three guesses of the next one, and what may follow the first two of them.
PARENTS = (-1, 0, 0, 0, 1, 1, 2, 4)
DEPTH = (0, 1, 1, 1, 2, 2, 2, 3)


class Device:
    """Lengths, tables and pool on the device, over the blocks that the planner's requests hold and others that it lends (a request that is never committed)."""

    def __init__(self, m, planner, texts, adapters, starts, growth):
        torch, bs = m.torch, m.bs
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to("cuda")
        rids, n = list(texts), [len(t) for t in texts.values()]
        tables = [planner.block_table(r) for r in rids]
        wide = np.full((len(rids), max(n) // bs + growth // bs + 3), -1, np.int32)
        for row, t in zip(wide, tables):
            row[: len(t)] = t
        self.tables, self.rows = i32(wide), len(rids) * len(PARENTS)
        lent = len(rids) * (growth // bs + 2)
        from .planner import Batch
        planner.admit(-1, np.zeros(lent * bs, np.int32), -1, NEVER, Batch(lent * bs, 1))
        self.pool = i32(planner.block_table(-1))
        # (one request's last blocks, taken from the end of the ring on, are its spare slots)
        self.spare = self.pool[-len(rids):].long() * bs
        self.lengths, self.lengths_out = i32(n), i32(n)
        self.kept = i32([len(t) for t in tables])                # what the planner gave stays the planner's
        self.adapters, self.starts = i32(adapters), i32(starts)
        self.state, self.state_out = i32([0, lent - len(rids), 0, 0, 0, 0]), i32([0] * 6)
        self.offsets = i32([0] * (len(rids) + 1))
        new = lambda dt=torch.int32: torch.zeros(self.rows, dtype=dt, device="cuda")
        self.seq, self.pos, self.aid, self.slot = new(), new(), new(), new(torch.int64)
        self.parents, self.depth = i32(PARENTS * len(rids)), torch.tensor(DEPTH, device="cuda")
        self.grow = i32([len(PARENTS)] * len(rids))
        self.dims = m.ab.make_step_dims(self.tables, bs, self.rows, self.pool, m.kc[0].shape[0])
        self.ab = m.ab

    def step(self, change):
        self.ab.alora_step_rows(self.lengths, change, self.kept, self.adapters, self.tables, self.pool, self.state, self.lengths_out, self.state_out, self.offsets,
                                self.seq, self.pos, self.aid, self.slot, self.dims)
        self.lengths, self.lengths_out = self.lengths_out, self.lengths
        self.state, self.state_out = self.state_out, self.state


def _layers(m, x, d, positions, attend):
    """Rows x through the layers, their keys and values to d's slots; attend(layer's q, K, V, layer) is the layer's attention."""
    torch, ab = m.torch, m.ab
    T, n_slots = x.shape[0], m.kc[0].shape[0]
    dims = ab.make_dims(ab.ALORA_BF16 if m.dt == torch.bfloat16 else ab.ALORA_F32, T, m.H, m.hq, m.hkv, m.d, m.adapters, m.rank, d.starts.shape[0], n_slots, d.seq,
                        positions)
    ws = ab.alloc_workspace(dims)
    q = torch.empty((T, m.hq * m.d), dtype=m.dt, device="cuda")
    heads = ab.make_heads_dims(q, q, None, m.kc[0], m.hq, m.hkv, m.d, rope=m.rope, interleaved=m.interleaved)
    for i, (l, kc, vc) in enumerate(zip(m.layers, m.kc, m.vc)):
        ab.alora_qkv_forward(x, d.aid, d.starts, l["W"], l["A"], l["B"], q, kc, vc, d.slot, m.bs, dims, ws)
        ab.alora_qk_norm_rope(q, q, None, kc, None, None, l["wq"], l["wk"], m.rope, positions, d.slot, heads)
        x = x + attend(q, kc, vc, i) @ l["O"]
    return x


def _tree_step(m, d, tokens):
    """tokens [sequences, drafts]; returns (accepted [sequences, drafts], the model's next token behind every draft)."""
    torch, ab = m.torch, m.ab
    S, N = tokens.shape
    context = d.lengths
    d.step(d.grow)
    mask = torch.empty((S * N, 1), dtype=torch.int64, device="cuda")
    positions = torch.empty((S * N,), dtype=torch.int32, device="cuda")
    ab.alora_tree_rows(d.parents, d.offsets, context, mask, positions)
    out = torch.empty((S * N, m.hq * m.d), dtype=m.dt, device="cuda")
    dims = ab.make_attn_dims(out, m.kc[0], d.tables, m.hq, m.hkv, m.d, m.bs)
    ws = torch.empty(ab.alora_tree_attention_workspace_bytes(dims, 1), dtype=torch.uint8, device="cuda")

    def attend(q, kc, vc, _):
        ab.alora_tree_attention(q, kc, vc, d.tables, d.offsets, context, mask, out, dims, ws)
        return out
    rows = _layers(m, m.emb[tokens.reshape(-1)], d, positions, attend)
    chosen = (rows @ m.head.T).argmax(-1).view(S, N)
    accepted = [torch.ones((S,), dtype=torch.bool, device="cuda")]
    for i in range(1, N):                                       # the first of a parent's children that is right
        p = PARENTS[i]
        right = accepted[p] & (tokens[:, i] == chosen[:, p])
        for j in range(1, i):
            if PARENTS[j] == p:
                right = right & ~accepted[j]
        accepted.append(right)
    return torch.stack(accepted, 1), chosen


def _keep_path(m, d, accepted, caches):
    """The accepted rows move together behind the context, the other places are given back."""
    torch, ab = m.torch, m.ab
    S, N = accepted.shape
    slot = d.slot.view(S, N)
    where = torch.where(accepted, d.depth, max(DEPTH) + 1)     # accepted drafts are one of a depth
    place = torch.full((S, max(DEPTH) + 2), -1, dtype=torch.int64, device="cuda").scatter_(1, where, slot)[:, :-1]
    there = place >= 0
    spare = d.spare[:, None] + torch.arange(max(DEPTH) + 1, device="cuda")
    none = torch.full_like(place, -1)
    ab.alora_cache_move_rows(place.reshape(-1), torch.where(there, spare, none).reshape(-1), None, None, caches)
    ab.alora_cache_move_rows(torch.where(there, spare, none).reshape(-1), torch.where(there, slot[:, : max(DEPTH) + 1], none).reshape(-1), None, None, caches)
    d.step((accepted.sum(1) - N).to(torch.int32))


def run(layers=4, prompt=1000, dtype="bf16", block_size=16, answer=40, seqs=3, seed=1) -> dict:
    import torch
    from . import planner as pl
    assert block_size > max(DEPTH)                             # a path fits a spare block
    growth = 3 * answer + 8 * len(PARENTS)
    lengths = [prompt, prompt // 3 + 1, *[prompt // 2 + 7 * i for i in range(seqs - 2)]]
    blocks = sum(-(-(n + growth) // block_size) + 4 for n in lengths) * 2 + seqs * (growth // block_size + 4)
    m = Model(layers, dtype, block_size, blocks, 128, False, 16 * ((prompt + growth) // 8 + 16), seed)
    ab, rng = m.ab, np.random.default_rng(seed)
    m.head = torch.from_numpy(rng.standard_normal((m.vocab, m.H)).astype(np.float32)).to("cuda", m.dt)
    p = pl.Planner(block_size, blocks)
    adapters, starts = [-1] * seqs, [NEVER] * seqs
    adapters[1], starts[1] = 0, lengths[1] // 2
    texts = {r: list(rng.integers(0, m.vocab, n).astype(np.int32)) for r, n in enumerate(lengths)}

    def prefill(rid, tokens, rid0):
        b = pl.Batch(len(tokens), 1)
        cached = p.admit(rid, np.array(tokens, np.int32), adapters[rid0], starts[rid0], b)
        y = m.step(p, b, [rid], np.array(tokens[cached:], np.int32))
        p.commit(rid)
        return y

    # -- 1: token by token
    first = [int((prefill(r, t, r)[-1] @ m.head.T).argmax()) for r, t in texts.items()]
    told = {r: [t] for r, t in enumerate(first)}
    for r in texts:                                            # (a conversation of its own: the first one's blocks stay as they are)
        prefill(100 + r, texts[r], r)
    for _ in range(answer):
        b = pl.Batch(seqs, seqs)
        for r in texts:
            p.append(100 + r, [told[r][-1]], b)
        rows = m.step(p, b, [100 + r for r in texts], np.array([told[r][-1] for r in texts], np.int32))
        for r, t in zip(texts, (rows @ m.head.T).argmax(-1).tolist()):
            told[r].append(t)
    # -- 2: with trees
    d = Device(m, p, texts, adapters, starts, growth)
    caches = ab.make_cache_dims(m.kc, m.vc, m.hkv, m.d, block_size)
    free0 = int(d.state[1])
    reference = torch.tensor([told[r] + [0] * 8 for r in texts], device="cuda")
    noise = torch.from_numpy(rng.integers(0, m.vocab, (answer, seqs, len(PARENTS)))).to("cuda")
    guess = torch.from_numpy(rng.random((answer, seqs, len(PARENTS))) < 0.6).to("cuda")
    at = torch.zeros((seqs,), dtype=torch.int64, device="cuda")   # how far each answer is
    known = torch.tensor(first, device="cuda")
    said = torch.full((seqs, answer * 4 + 8), -1, dtype=torch.int64, device="cuda")
    depth, steps = d.depth, 0
    while steps < answer // 2:
        right = reference.gather(1, (at[:, None] + depth).clamp(max=reference.shape[1] - 1))
        tokens = torch.where(guess[steps], right, noise[steps])
        tokens[:, 0] = known
        accepted, chosen = _tree_step(m, d, tokens)
        said.scatter_(1, torch.where(accepted, at[:, None] + depth, said.shape[1] - 1), tokens)
        last = (accepted * (depth + 1)).argmax(1)
        known = chosen.gather(1, last[:, None])[:, 0]
        _keep_path(m, d, accepted, caches)
        at = at + accepted.sum(1)
        steps += 1
    at, said = at.tolist(), said.cpu().numpy()
    res = dict(steps=steps, tokens=sum(at), same_as_told=[int(np.argmin(np.append(said[r][: at[r]] == told[r][: at[r]] if at[r] <= len(told[r]) else said[r][: len(told[r])] == told[r], False)))
                                                        for r in texts])
    res["told"] = [min(a, answer + 1) for a in at]
    res["lengths"] = bool((d.lengths.cpu().numpy() == [len(t) + a for t, a in zip(texts.values(), at)]).all())
    held = sum(-(-(len(t) + a) // block_size) - len(p.block_table(r)) for (r, t), a in zip(texts.items(), at))
    res["blocks_kept"] = bool(int(d.state[1]) == free0 - held)
    # what a computation from scratch of the same text would have chosen, and what it leaves in the cache
    gap = size = key_off = value_off = 0.0
    kept = m.kc, m.vc, m.cache
    final = {r: np.array(texts[r] + said[r][: at[r]].tolist(), np.int32) for r in texts}
    tables, places = d.tables.cpu().numpy(), {}
    for r, text in final.items():
        m.new_caches(len(text) // block_size + 1)
        other, b = pl.Planner(block_size, len(text) // block_size + 1), pl.Batch(len(text), 1)
        other.admit(1, text, adapters[r], starts[r], b)
        logits = (m.step(other, b, [1], text) @ m.head.T).float()
        n, j = len(texts[r]), np.arange(len(text))
        took = logits[n - 1: -1].gather(1, torch.from_numpy(text[n:].astype(np.int64)).to("cuda")[:, None])[:, 0]
        gap, size = max(gap, float((logits[n - 1: -1].amax(-1) - took).max())), max(size, float(logits.abs().max()))
        places[r] = torch.from_numpy(tables[r][j // block_size].astype(np.int64) * block_size + j % block_size).to("cuda")
        k, v = m.rows_of(other, 1, len(text), 0)
        key_off, value_off = max(key_off, _off(kept[0][0][places[r]], k)), max(value_off, _off(kept[1][0][places[r]], v))
        other.close()
    m.kc, m.vc, m.cache = kept
    res.update(choice_gap=gap / size, key_off=key_off, value_off=value_off)
    # -- 3: over selected blocks
    n_blocks = m.kc[0].shape[0] // block_size
    bounds = [(torch.zeros((n_blocks, m.hkv, 2, m.d), dtype=torch.int8, device="cuda"), torch.zeros((n_blocks, m.hkv), device="cuda")) for _ in m.layers]
    for (b, s), kc in zip(bounds, m.kc):
        for slots in places.values():
            ab.alora_block_bounds(kc, slots, b, s, ab.make_bounds_dims(kc, slots, m.hkv, m.d, block_size))
    one = torch.ones((seqs,), dtype=torch.int32, device="cuda")
    d.step(one)
    d.seq, d.pos, d.aid, d.slot = (x[:seqs].contiguous() for x in (d.seq, d.pos, d.aid, d.slot))
    x = m.emb[known]
    out = torch.empty((seqs, m.hq * m.d), dtype=m.dt, device="cuda")
    dims = ab.make_attn_dims(out, m.kc[0], d.tables, m.hq, m.hkv, m.d, block_size)
    first_layer = []

    def over(budget):
        chosen = torch.empty((seqs, m.hkv, budget), dtype=torch.int32, device="cuda")
        ws = torch.empty(max(16, ab.alora_block_select_workspace_bytes(dims), ab.alora_selected_attention_workspace_bytes(dims, budget)), dtype=torch.uint8, device="cuda")

        def attend(q, kc, vc, i):
            ab.alora_block_bounds(kc, d.slot, *bounds[i], ab.make_bounds_dims(kc, d.slot, m.hkv, m.d, block_size))
            ab.alora_block_select(q, *bounds[i], d.tables, d.seq, d.pos, chosen, 1, 2, dims, ws)
            ab.alora_selected_attention(q, kc, vc, d.tables, d.seq, d.pos, chosen, out, dims, ws)
            if i == 0:
                first_layer.append(out.clone())
            return out
        return _layers(m, x, d, d.pos, attend)

    def whole(q, kc, vc, i):
        ab.alora_paged_attention(q, kc, vc, d.tables, d.seq, d.pos, out, dims)
        if i == 0:
            first_layer.append(out.clone())
        return out
    full = _layers(m, x, d, d.pos, whole)
    most = int(d.lengths.max()) // block_size + 1
    res["all_blocks_off"] = _off(over(most), full)
    res["all_blocks_attention_off"] = _off(first_layer[1], first_layer[0])      # (of the same queries)
    res["some_blocks"], res["of_blocks"] = max(4, most // 4), most
    res["some_blocks_finite"] = bool(torch.isfinite(over(res["some_blocks"])).all())
    p.close()
    return res


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--answer", type=int, default=40)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    args = ap.parse_args()
    print(json.dumps(run(args.layers, args.prompt, args.dtype, answer=args.answer)))


if __name__ == "__main__":
    main()
