#!/usr/bin/env python3
"""One conversation through a few layers whose query and key heads are normalised, with angles scaled for long contexts: what
alora_heads.h and alora_cache.h are for, next to the planner, the projection and the reader.

  1. tables of the scaled angles are computed on the device;
  2. the base model reads a prompt and answers (projection, norm and rotation in place on the cache, reader; every layer);
  3. an adapter is invoked on the conversation, which goes on besides: a fork shares the full blocks and copies the partial one;
  4. a turn is dropped from the middle: the rows behind move up, their keys turned by the shift;
  5. the pool is made smaller: blocks behind its new end move;
  6. the norms' weights of a layer take a few training steps towards other heads (the backward pass).

Synthetic data.  Checks itself (the fork against the same request computed from scratch, the dropped rows of the first layer, whose
keys do not see other tokens, against theirs from scratch, answers before and after the pool became smaller, the falling loss) and prints one
JSON line.

    python -m paper_2512_17910_amd.conversation [--layers 4] [--prompt 1000] [--dtype bf16|f32] [--interleaved]
"""
from __future__ import annotations

import argparse
import json
import time

import numpy as np

NEVER = 1 << 30


class Model:
    """Weights of the layers, the paged caches, and the calls of a step."""

    def __init__(self, layers, dtype, block_size, n_blocks, rotary_dim, interleaved, positions, seed=1):
        import torch
        from . import binding as ab
        self.ab, self.torch = ab, torch
        self.H, self.hq, self.hkv, self.d, self.bs = 512, 8, 2, 128, block_size
        self.rank, self.adapters, self.vocab = 16, 2, 211
        self.interleaved = interleaved
        dt = self.dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rnd = lambda shape, std, mean=0.0: (torch.randn(shape, device="cuda", generator=g) * std + mean).to(dt)
        nq, nkv = self.hq * self.d, self.hkv * self.d
        n = nq + 2 * nkv
        self.emb = rnd((self.vocab, self.H), 1.0)
        self.layers = [dict(W=rnd((self.H, n), self.H ** -0.5), A=[rnd((self.H, self.rank), self.H ** -0.5) for _ in range(self.adapters)],
                            B=[rnd((self.rank, n), self.rank ** -0.5) for _ in range(self.adapters)], O=rnd((nq, self.H), nq ** -0.5),
                            wq=rnd((self.d,), 0.2, 1.0), wk=rnd((self.d,), 0.2, 1.0)) for _ in range(layers)]
        self.rope = tuple(torch.empty((positions, rotary_dim // 2), device="cuda") for _ in range(2))
        # (the magnitude goes into the scores' scale here: cached keys can be turned with the same tables)
        ab.alora_rope_tables(*self.rope, ab.make_rope_spec(rotary_dim, 500000.0, "by_parts", 16.0, original=positions // 16, low=1.0, high=32.0))
        self.new_caches(n_blocks)

    def new_caches(self, n_blocks):
        shape = (n_blocks * self.bs, self.hkv * self.d)
        self.kc, self.vc = ([self.torch.zeros(shape, dtype=self.dt, device="cuda") for _ in self.layers] for _ in range(2))
        self.cache = self.ab.make_cache_dims(self.kc, self.vc, self.hkv, self.d, self.bs)

    def step(self, planner, batch, rids, tokens):
        """The batch's rows through the layers; returns the last layer's rows."""
        ab, torch = self.ab, self.torch
        pos, seg, aid, slot, start = (torch.from_numpy(a.copy()).to("cuda") for a in batch.rows())
        tables = [planner.block_table(r) for r in rids]
        wide = np.zeros((len(rids), max(map(len, tables))), np.int32)
        for row, t in zip(wide, tables):
            row[: len(t)] = t
        bt = torch.from_numpy(wide).to("cuda")
        x = self.emb[torch.as_tensor(tokens, device="cuda")]
        T, n_slots = x.shape[0], self.kc[0].shape[0]
        dims = ab.make_dims(ab.ALORA_BF16 if self.dt == torch.bfloat16 else ab.ALORA_F32, T, self.H, self.hq, self.hkv, self.d, self.adapters,
                            self.rank, len(rids), n_slots, seg, pos)
        ws = ab.alloc_workspace(dims)
        q = torch.empty((T, self.hq * self.d), dtype=self.dt, device="cuda")
        out = torch.empty_like(q)
        heads = ab.make_heads_dims(q, q, None, self.kc[0], self.hq, self.hkv, self.d, rope=self.rope, interleaved=self.interleaved)
        attn = ab.make_attn_dims(q, self.kc[0], bt, self.hq, self.hkv, self.d, self.bs)
        for l, kc, vc in zip(self.layers, self.kc, self.vc):
            ab.alora_qkv_forward(x, aid, start, l["W"], l["A"], l["B"], q, kc, vc, slot, self.bs, dims, ws)
            ab.alora_qk_norm_rope(q, q, None, kc, None, None, l["wq"], l["wk"], self.rope, pos, slot, heads)
            ab.alora_paged_attention(q, kc, vc, bt, seg, pos, out, attn)
            x = x + out @ l["O"]
        return x

    def rows_of(self, planner, rid, n, layer):
        t, p = planner.block_table(rid), np.arange(n)
        at = self.torch.from_numpy(t[p // self.bs].astype(np.int64) * self.bs + p % self.bs).to("cuda")
        return self.kc[layer][at], self.vc[layer][at]


def _off(a, b) -> float:
    """Largest difference relative to the largest value."""
    a, b = a.double(), b.double()
    return float((a - b).abs().max() / b.abs().max())


def run(layers=4, prompt=1000, dtype="bf16", block_size=16, rotary_dim=128, interleaved=False, seed=1) -> dict:
    import torch
    from . import planner as pl
    positions = 16 * (prompt // 8 + 16)
    n_blocks = 6 * (prompt // block_size + 8)
    m = Model(layers, dtype, block_size, n_blocks, rotary_dim, interleaved, positions, seed)
    ab, p = m.ab, pl.Planner(block_size, n_blocks)
    rng = np.random.default_rng(seed)
    tok = lambda n: rng.integers(0, m.vocab, n).astype(np.int32)
    res, texts = {}, {}

    def admit(rid, tokens):
        b = pl.Batch(len(tokens), 1)
        cached = p.admit(rid, tokens, -1, NEVER, b)
        m.step(p, b, [rid], tokens[cached:])
        p.commit(rid)
        texts[rid] = list(tokens)

    def from_scratch(tokens, adapter=-1, start=NEVER):
        """The last layer's rows and the first layer's keys and values of a request that finds nothing in the cache."""
        kept = m.kc, m.vc, m.cache
        blocks = len(tokens) // block_size + 1
        m.new_caches(blocks)
        other, b = pl.Planner(block_size, blocks), pl.Batch(len(tokens), 1)
        tokens = np.array(tokens, np.int32)
        other.admit(1, tokens, adapter, start, b)
        y = m.step(other, b, [1], tokens)
        kv = m.rows_of(other, 1, len(tokens), 0)
        other.close()
        m.kc, m.vc, m.cache = kept
        return y, *kv

    def answer(rids, news):
        b = pl.Batch(sum(map(len, news)), len(rids))
        for r, new in zip(rids, news):
            p.append(r, new, b)
            texts[r] += list(new)
        y = m.step(p, b, rids, np.concatenate(news))
        for r in rids:
            p.commit(r)
        return y

    admit(9, tok(5 * block_size + 1))         # another request, over before the pool is made smaller
    admit(1, tok(prompt))
    for _ in range(3):
        answer([1], [tok(1)])
    # -- the adapter is invoked; the conversation goes on
    n = len(texts[1])
    src, dst = p.fork(1, 2, 0, n)
    ab.alora_cache_copy_blocks(src, dst, m.cache)
    texts[2] = list(texts[1])
    forked = answer([1, 2], [tok(5), tok(21)])[5:]
    scratch = from_scratch(texts[2], 0, n)[0]
    res["forked_blocks_shared"] = int((p.block_table(1)[: n // block_size] == p.block_table(2)[: n // block_size]).sum())
    res["fork_off"] = _off(forked, scratch[-21:])
    # -- a turn is dropped
    first, dropped = prompt // 3, prompt // 4 + 1
    src, dst, shift = p.drop(1, first, dropped)
    moved = [torch.from_numpy(a).to("cuda") for a in (src, dst, shift)]
    assert ab.alora_cache_move_rows_validate(*moved, m.rope, m.cache) == ab.ALORA_OK
    torch.cuda.synchronize()
    t = time.perf_counter()
    ab.alora_cache_move_rows(*moved, m.rope, m.cache, interleaved=interleaved)
    torch.cuda.synchronize()
    res["moved_rows"], res["move_ms"] = len(src), (time.perf_counter() - t) * 1e3
    del texts[1][first: first + dropped]
    k, v = m.rows_of(p, 1, len(texts[1]), 0)
    _, k_new, v_new = from_scratch(texts[1])
    res["drop_key_off"], res["drop_value_off"] = _off(k, k_new), _off(v, v_new)
    answer([1], [tok(2)])
    # -- the pool is made smaller
    p.finish(9)
    probe = tok(1)

    def look():
        p_rows = pl.Batch(1, 1)
        p.append(2, probe, p_rows)
        return m.step(p, p_rows, [2], probe)
    before = look()
    moved = [torch.from_numpy(a).to("cuda") for a in p.drop(2, len(texts[2]), 1)]     # the probe again: what its block holds moves, unturned
    ab.alora_cache_move_rows(*moved, m.rope, m.cache, interleaved=interleaved)
    used = n_blocks - p.free_blocks()
    src, dst = p.compact(used + 1)
    ab.alora_cache_copy_blocks(src, dst, m.cache)
    keep = (used + 1) * block_size
    m.kc, m.vc = ([c[:keep].clone() for c in cs] for cs in (m.kc, m.vc))
    m.cache = ab.make_cache_dims(m.kc, m.vc, m.hkv, m.d, block_size)
    res["compacted_blocks"], res["blocks"], res["blocks_before"] = len(src), used + 1, n_blocks
    res["same_answer"] = bool(torch.equal(before, look()))
    # -- training steps of a layer's norms
    res["loss"] = _train(m, tok(333), interleaved)
    p.close()
    return res


def _train(m, tokens, interleaved, steps=5):
    """Heads of a layer towards those of other norm weights: loss = mean square of the difference."""
    torch, ab = m.torch, m.ab
    l, T = m.layers[0], len(tokens)
    nq, nkv = m.hq * m.d, m.hkv * m.d
    y = m.emb[torch.as_tensor(tokens, device="cuda")] @ l["W"]              # q | k | v
    q, k = y[:, :nq], y[:, nq: nq + nkv]
    pos, slot = torch.arange(T, dtype=torch.int32, device="cuda"), torch.arange(T, device="cuda")
    out = [torch.empty((T, w), dtype=m.dt, device="cuda") for w in (nq, nkv)]
    grads = [torch.empty_like(o) for o in out]
    dims = ab.make_heads_dims(q, out[0], k, out[1], m.hq, m.hkv, m.d, rope=m.rope, interleaved=interleaved)
    back = ab.make_heads_dims(q, out[0], k, out[1], m.hq, m.hkv, m.d, rope=m.rope, interleaved=interleaved, dq=grads[0], dk=grads[1])
    ws = torch.empty(max(16, ab.alora_qk_norm_rope_workspace_bytes(back)), dtype=torch.uint8, device="cuda")
    w = [torch.ones(m.d, device="cuda") for _ in range(2)]                  # trained in 32 bits
    dw = [torch.empty(m.d, device="cuda") for _ in range(2)]
    heads = lambda wq, wk: ab.alora_qk_norm_rope(q, out[0], k, out[1], None, None, wq, wk, m.rope, pos, slot, dims)
    heads(l["wq"], l["wk"])
    target = [o.clone() for o in out]
    losses = []
    for _ in range(steps):
        wq, wk = (x.to(m.dt) for x in w)
        heads(wq, wk)
        diff = [o.float() - t.float() for o, t in zip(out, target)]
        losses.append(float(sum((x * x).mean() for x in diff)))
        g = [(2.0 * x / x.numel()).to(m.dt) for x in diff]
        ab.alora_qk_norm_rope_backward(q, g[0], grads[0], k, g[1], grads[1], wq, wk, dw[0], dw[1], m.rope, pos, back, ws)
        for x, dx in zip(w, dw):
            x -= 0.3 * m.d * dx
    return losses


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--interleaved", action="store_true")
    args = ap.parse_args()
    print(json.dumps(run(args.layers, args.prompt, args.dtype, interleaved=args.interleaved)))


if __name__ == "__main__":
    main()
