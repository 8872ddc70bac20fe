"""What is timed of the operators between the projection and the reader, and of the cache's pages.

Five kinds of work, each one call of paper_2512_17910_amd.binding:

  heads       norm of every query and key head and rotary embedding in one pass (alora_qk_norm_rope): "cache" works in
              place, on the queries and on the rows of the paged cache that the projection has just written; "buffer"
              reads a fused q | k | v buffer and writes the queries and both caches.
  heads-back  its backward pass (alora_qk_norm_rope_backward): gradients of queries and keys, and of the two norms' weights.
  tables      cosines and sines of a range of positions, scaled for long contexts (alora_rope_tables).
  blocks      copies of cache blocks over all layers (alora_cache_copy_blocks): a fork's partial block, a pool that is made
              dense, blocks that are cleared.
  rows        token rows moved to other slots over all layers, keys turned by the shift of their positions
              (alora_cache_move_rows): tokens dropped from the middle of conversations.

Shapes are those of the repository's configurations (32 / 8 and 64 / 8 heads of 128, the small fp32 layer with 4 / 2 heads
of 64) and generic ones in between; blocks of 16 tokens unless a case says otherwise.  Values: queries, keys and values as a
projection leaves them, N(0, 1) times a scale of each head's own; norm weights around 1; cached values N(0, 1).
"""
import math

import numpy as np
import torch

own = False             # the tools set it: run() calls the library's operators, not their plain forms

MAX_POS = 32768         # rows of the rotary tables that a model of these shapes keeps
EPS = 1e-6


def listed():
    return [
        # one conversation is being answered: one token, its key in the cache.  The smallest call: launches and the host count
        {"name": "heads-decode-1", "kind": "heads", "form": "cache", "dtype": "bf16", "rows": 1, "hq": 32, "hkv": 8, "d": 128, "rot": 128,
         "interleaved": False, "norm": True, "decode": True, "pad": 0},
        # a busy server: 256 requests decode together
        {"name": "heads-decode-256", "kind": "heads", "form": "cache", "dtype": "bf16", "rows": 256, "hq": 32, "hkv": 8, "d": 128, "rot": 128,
         "interleaved": False, "norm": True, "decode": True, "pad": 0},
        # a step of chunked prefill in reference precision, heads of an odd size of which the first part is turned
        {"name": "heads-chunk-777-f32", "kind": "heads", "form": "buffer", "dtype": "f32", "rows": 777, "hq": 12, "hkv": 4, "d": 80, "rot": 20,
         "interleaved": False, "norm": True, "decode": False, "pad": 0},
        # a large prefill step of the large model, neighbours paired, half of each head turned
        {"name": "heads-prefill-8192", "kind": "heads", "form": "buffer", "dtype": "bf16", "rows": 8192, "hq": 64, "hkv": 8, "d": 128, "rot": 64,
         "interleaved": True, "norm": True, "decode": False, "pad": 0},
        # an adapter is trained on short ragged texts, the small layer in reference precision
        {"name": "back-613-f32", "kind": "heads-back", "dtype": "f32", "rows": 613, "hq": 4, "hkv": 2, "d": 64, "rot": 64,
         "interleaved": False, "norm": True},
        # an adapter of an ordinary layer is trained: 4096 tokens
        {"name": "back-4096", "kind": "heads-back", "dtype": "bf16", "rows": 4096, "hq": 32, "hkv": 8, "d": 128, "rot": 128,
         "interleaved": False, "norm": True},
        # a model that turns half of each head is loaded for short contexts, its positions pressed together
        {"name": "tables-2048", "kind": "tables", "rows": 2048, "rot": 64, "first": 0, "base": 10000.0, "scaling": "linear", "factor": 4.0,
         "original": 2048, "low": 1.0, "high": 32.0, "magnitude": 1.0},
        # a model is loaded for contexts of 131072 tokens, scaled by parts
        {"name": "tables-131072", "kind": "tables", "rows": 131072, "rot": 128, "first": 0, "base": 500000.0, "scaling": "by_parts", "factor": 16.0,
         "original": 8192, "low": 1.0, "high": 32.0, "magnitude": 1.2772588722239782},
        # an adapter is invoked on a conversation that goes on besides: the partial block of the fork, over all layers
        {"name": "blocks-fork-1", "kind": "blocks", "dtype": "bf16", "layers": 32, "blocks": 256, "pairs": 1, "clears": 0, "hkv": 8, "d": 128, "bs": 16},
        # a pool is made dense before it is made smaller: many blocks move, over a group of layers
        {"name": "blocks-compact-1000", "kind": "blocks", "dtype": "bf16", "layers": 8, "blocks": 2300, "pairs": 1000, "clears": 13, "hkv": 8, "d": 128,
         "bs": 16},
        # a turn is dropped from the middle of a conversation of the small layer: what follows moves up
        {"name": "rows-211-f32", "kind": "rows", "dtype": "f32", "layers": 2, "seqs": 1, "rows": 211, "hkv": 2, "d": 64, "rot": 64,
         "interleaved": False, "bs": 16},
        # a few long conversations lose their oldest turns behind the first instructions
        {"name": "rows-9001", "kind": "rows", "dtype": "bf16", "layers": 16, "seqs": 3, "rows": 9001, "hkv": 8, "d": 128, "rot": 128,
         "interleaved": False, "bs": 16},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    u = rng.random()
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    e = 2 if dtype == "bf16" else 4
    hkv = rng.choice([1, 2, 4, 8, 8, 8])
    d = rng.choice([64, 128, 128, 128, 32, 80, 96, 112, 192, 256])
    rot = rng.choice([d, d, d, d // 2, 2 * (d // 8)])
    if u < 0.4:
        hq = hkv * rng.choice([1, 2, 3, 4, 4, 7, 8])
        rows = _log_int(rng, 1, 8192)
        rows = min(rows, (8192 * 80 * 128 * 2) // ((hq + 2 * hkv) * d * e))        # no more data than the largest listed case
        decode = rows <= 256 and rng.random() < 0.7
        form, norm = rng.choice(["cache", "cache", "buffer"]), rng.random() < 0.8
        return {"kind": "heads", "form": form, "dtype": dtype, "rows": rows, "hq": hq, "hkv": hkv, "d": d,
                "rot": rng.choice([rot, rot, rot, 0]) if norm else rot, "interleaved": rng.random() < 0.4, "norm": norm, "decode": decode,
                "pad": rng.randint(0, rows // 4) if form == "cache" and rng.random() < 0.3 else 0}
    if u < 0.6:
        hq = hkv * rng.choice([1, 2, 3, 4, 4, 7, 8])
        rows = min(_log_int(rng, 1, 4096), (4096 * 40 * 128 * 2) // ((hq + hkv) * d * e))
        return {"kind": "heads-back", "dtype": dtype, "rows": rows, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "interleaved": rng.random() < 0.4,
                "norm": rng.random() < 0.85}
    if u < 0.7:
        return {"kind": "tables", "rows": _log_int(rng, 16, 131072), "rot": rng.choice([16, 20, 32, 64, 96, 128]),
                "first": rng.choice([0, 0, rng.randint(1, 900000)]), "base": rng.choice([10000.0, 500000.0, 1000000.0]), "scaling": rng.choice(["none", "linear", "by_parts", "by_parts"]),
                "factor": rng.choice([2.0, 4.0, 8.0, 16.0, 40.0]), "original": rng.choice([2048, 4096, 8192, 32768]), "low": 1.0,
                "high": rng.choice([4.0, 32.0]), "magnitude": rng.choice([1.0, 1.0, 1.1386294361119891])}
    if u < 0.85:
        bs, layers = rng.choice([16, 16, 16, 32, 64, 8]), rng.choice([1, 2, 4, 8, 16, 32])
        block = 2 * layers * bs * hkv * d * e                                      # bytes of one block in all layers
        pairs = max(1, min(_log_int(rng, 1, 1000), 500_000_000 // block))
        return {"kind": "blocks", "dtype": dtype, "layers": layers, "blocks": min(2 * pairs + rng.randint(1, 300), max(2 * pairs + 1, 1_200_000_000 // block)),
                "pairs": pairs, "clears": rng.randint(0, pairs // 10), "hkv": hkv, "d": d, "bs": bs}
    layers, seqs = rng.choice([1, 2, 4, 8, 16]), rng.randint(1, 4)
    rows = max(seqs, min(_log_int(rng, 1, 9001), 590_000_000 // (2 * layers * hkv * d * e)))
    return {"kind": "rows", "dtype": dtype, "layers": layers, "seqs": seqs, "rows": rows, "hkv": hkv, "d": d, "rot": rng.choice([rot, rot, rot, 0]),
            "interleaved": rng.random() < 0.4, "bs": rng.choice([16, 16, 32, 64])}


# ---- inputs -------------------------------------------------------------------------------------
def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


class _Values:
    """Normally distributed tensors, one generator on the GPU."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = dtype

    def __call__(self, shape, std=1.0, mean=0.0):
        return (torch.randn(shape, device="cuda", generator=self.g, dtype=torch.float32) * std + mean).to(self.dtype)

    def rows(self, t, heads, d):
        """Rows of heads, each head with a scale of its own, from 0.1 to 10."""
        scale = 10.0 ** (2.0 * torch.rand((heads, 1), device="cuda", generator=self.g) - 1.0)
        return self((t, heads, d), scale).view(t, heads * d)


def _rope_tables(rot, base=10000.0):
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * (base ** (-2.0 * i / rot))[None, :]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _cut(rng, total, parts):
    """`total` rows cut into `parts` ragged pieces, none empty."""
    cuts = np.sort(rng.choice(np.arange(1, total), size=parts - 1, replace=False)) if parts > 1 else np.zeros(0, np.int64)
    return np.diff(np.concatenate([[0], cuts, [total]])).astype(np.int64)


def _positions(rng, rows, decode):
    """Positions and slots of the rows of a batch: a row per sequence, or pieces of a few sequences; blocks of 16 dealt at random."""
    lens = np.ones(rows, np.int64) if decode else _cut(rng, rows, min(5, rows))
    first = np.array([rng.integers(0, MAX_POS - n + 1) for n in lens])
    pos = np.concatenate([np.arange(f, f + n) for f, n in zip(first, lens)])
    b0, b1 = first // 16, (first + lens - 1) // 16 + 1
    blocks = rng.permutation(rows // 16 + 2 * len(lens) + 66)       # (a size that the row count gives, other blocks among them)
    seg, at = np.repeat(np.arange(len(lens)), lens), np.concatenate([[0], np.cumsum(b1 - b0)])[:-1]
    return pos.astype(np.int32), blocks[at[seg] + pos // 16 - b0[seg]].astype(np.int64) * 16 + pos % 16, 16 * len(blocks)


class _Heads:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
        pos, slot, n_slots = _positions(rng, t, case["decode"])
        slot[t - case["pad"]:] = -1                                 # a recorded batch that is not full
        self.pos, self.slot = _dev(pos), _dev(slot)
        self.rope = _rope_tables(case["rot"]) if case["rot"] else None
        self.wq, self.wk = ((values((d,), 0.2, 1.0) for _ in range(2)) if case["norm"] else (None, None))
        self.kc, self.vc = values((n_slots, hkv * d)), values((n_slots, hkv * d))
        if case["form"] == "cache":                                 # the projection has stored q and, at the slots, k and v
            self.q = self.q_out = values.rows(t, hq, d)
            self.k = self.v = None
            real = t - case["pad"]
            self.kc[self.slot[:real]] = values.rows(real, hkv, d)
        else:
            y = torch.cat((values.rows(t, hq, d), values.rows(t, hkv, d), values.rows(t, hkv, d)), 1)
            self.q, self.k, self.v = y[:, : hq * d], y[:, hq * d: (hq + hkv) * d], y[:, (hq + hkv) * d:]
            self.q_out = torch.empty((t, hq * d), dtype=y.dtype, device="cuda")
        self.dims = None                                            # the library's description of the call, made in the first pass

    def _own(self, case):
        from paper_2512_17910_amd import binding as ab
        if self.dims is None:
            self.dims = ab.make_heads_dims(self.q, self.q_out, self.k, self.kc, case["hq"], case["hkv"], case["d"], rope=self.rope,
                                           interleaved=case["interleaved"], norm=case["norm"], eps=EPS, v=self.v, v_out=self.vc)
        ab.alora_qk_norm_rope(self.q, self.q_out, self.k, self.kc, self.v, self.vc if self.v is not None else None, self.wq, self.wk, self.rope,
                              self.pos, self.slot, self.dims)
        return self.q_out, self.kc, self.vc

    def run(self, case):
        if own:
            return self._own(case)
        t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
        c, s = (x[self.pos.long()][:, None, :] for x in self.rope) if self.rope else (None, None)
        self.q_out.copy_(_plain_heads(self.q.view(t, hq, d), self.wq, c, s, case).view(t, hq * d))
        if self.k is None:
            new = _plain_heads(self.kc[self.slot.clamp(min=0)].view(t, hkv, d), self.wk, c, s, case).view(t, hkv * d)
            if case["pad"]:
                keep = self.slot >= 0
                self.kc[self.slot[keep]] = new[keep]
            else:
                self.kc[self.slot] = new
        else:
            self.kc[self.slot] = _plain_heads(self.k.view(t, hkv, d), self.wk, c, s, case).view(t, hkv * d)
            self.vc[self.slot] = self.v
        return self.q_out, self.kc, self.vc


class _HeadsBack:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
        self.pos = _dev(_positions(rng, t, False)[0])
        self.rope = _rope_tables(case["rot"])
        self.wq, self.wk = ((values((d,), 0.2, 1.0) for _ in range(2)) if case["norm"] else (None, None))
        y = torch.cat((values.rows(t, hq, d), values.rows(t, hkv, d), values((t, hkv * d))), 1)
        dy = torch.empty_like(y)                                    # gradient of the fused buffer; v's part is not this operator's
        cut = (slice(0, hq * d), slice(hq * d, (hq + hkv) * d))
        self.q, self.k = (y[:, c] for c in cut)
        self.dq, self.dk = (dy[:, c] for c in cut)
        self.dq_out, self.dk_out = values((t, hq * d)), values((t, hkv * d))
        self.dwq, self.dwk = ((torch.empty((d,), device="cuda") for _ in range(2)) if case["norm"] else (None, None))
        self.dims = self.ws = None

    def _own(self, case):
        from paper_2512_17910_amd import binding as ab
        if self.dims is None:
            self.dims = ab.make_heads_dims(self.q, self.dq_out, self.k, self.dk_out, case["hq"], case["hkv"], case["d"], rope=self.rope,
                                           interleaved=case["interleaved"], norm=case["norm"], eps=EPS)
            self.ws = torch.empty(max(16, ab.alora_qk_norm_rope_workspace_bytes(self.dims)), dtype=torch.uint8, device="cuda")
        ab.alora_qk_norm_rope_backward(self.q, self.dq_out, self.dq, self.k, self.dk_out, self.dk, self.wq, self.wk, self.dwq, self.dwk, self.rope,
                                       self.pos, self.dims, self.ws)
        return self.dq, self.dk, self.dwq, self.dwk

    def run(self, case):
        if own:
            return self._own(case)
        t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
        c, s = (x[self.pos.long()][:, None, :] for x in self.rope)
        dq, dwq = _plain_heads_back(self.q.view(t, hq, d), self.dq_out.view(t, hq, d), self.wq, c, s, case)
        dk, dwk = _plain_heads_back(self.k.view(t, hkv, d), self.dk_out.view(t, hkv, d), self.wk, c, s, case)
        self.dq.copy_(dq.view(t, hq * d))
        self.dk.copy_(dk.view(t, hkv * d))
        return self.dq, self.dk, dwq, dwk


class _Tables:
    def __init__(self, case, seed):
        # a seed is another place: the first position, or where that is 0 the base, is the seed's own
        rng = np.random.default_rng(seed)
        self.first = case["first"] + int(rng.integers(0, 4096)) if case["first"] else 0
        self.base = case["base"] * float(rng.uniform(1.0, 1.01))
        self.cos, self.sin = (torch.empty((case["rows"], case["rot"] // 2), device="cuda") for _ in range(2))
        self.spec = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.spec is None:
                self.spec = ab.make_rope_spec(case["rot"], self.base, case["scaling"], case["factor"], case["original"], case["low"], case["high"],
                                              case["magnitude"])
            ab.alora_rope_tables(self.cos, self.sin, self.spec, self.first)
            return self.cos, self.sin
        i = torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64)
        theta = self.base ** (-2.0 * i / case["rot"])
        if case["scaling"] == "linear":
            theta = theta / case["factor"]
        elif case["scaling"] == "by_parts":
            g = ((case["original"] * theta / (2.0 * math.pi) - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
            theta = theta * ((1.0 - g) / case["factor"] + g)
        angle = torch.arange(self.first, self.first + case["rows"], device="cuda", dtype=torch.float64)[:, None] * theta[None, :]
        self.cos.copy_(torch.cos(angle) * case["magnitude"])
        self.sin.copy_(torch.sin(angle) * case["magnitude"])
        return self.cos, self.sin


class _Blocks:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        self.caches = values((case["layers"], 2, case["blocks"], case["bs"] * case["hkv"] * case["d"]))
        perm = rng.permutation(case["blocks"]).astype(np.int32)
        self.src, self.dst = perm[: case["pairs"]].copy(), perm[case["pairs"]: 2 * case["pairs"]].copy()   # the planner's answer: host arrays
        self.src[case["pairs"] - case["clears"]:] = -1
        self.dims = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                layers = self.caches.view(case["layers"], 2, case["blocks"] * case["bs"], case["hkv"] * case["d"])
                self.dims = ab.make_cache_dims([y[0] for y in layers], [y[1] for y in layers], case["hkv"], case["d"], case["bs"])
            ab.alora_cache_copy_blocks(self.src, self.dst, self.dims)
            return self.caches
        n = case["pairs"] - case["clears"]
        src, dst = torch.from_numpy(self.src).long().to("cuda"), torch.from_numpy(self.dst).long().to("cuda")
        self.caches[:, :, dst[:n]] = self.caches[:, :, src[:n]]
        if case["clears"]:
            self.caches[:, :, dst[n:]] = 0
        return self.caches


class _Rows:
    def __init__(self, case, seed):
        rng, values = np.random.default_rng(seed), _Values(seed, _dtype(case))
        n, bs = case["rows"], case["bs"]
        lens = _cut(rng, n, min(case["seqs"], n))
        drop = rng.integers(1, 4097, len(lens))                     # tokens that each sequence loses in front of its rows
        first = rng.integers(0, 129, len(lens)) + drop              # old position of the first row that moves
        seg, pos = np.repeat(np.arange(len(lens)), lens), np.concatenate([np.arange(f, f + m) for f, m in zip(first, lens)])
        new = pos - drop[seg]
        spare = n // bs + 2 * len(lens) + 2
        perm = rng.permutation(2 * spare)

        def slots(p, blocks):
            b0 = np.array([p[seg == s].min() // bs for s in range(len(lens))])
            b1 = np.array([p[seg == s].max() // bs + 1 for s in range(len(lens))])
            at = np.concatenate([[0], np.cumsum(b1 - b0)])[:-1]
            return blocks[at[seg] + p // bs - b0[seg]].astype(np.int64) * bs + p % bs

        self.src, self.dst = _dev(slots(pos, perm[:spare])), _dev(slots(new, perm[spare:]))
        self.shift = _dev((new - pos).astype(np.int32))
        self.rope = _rope_tables(case["rot"]) if case["rot"] else None
        self.caches = values((case["layers"], 2, 2 * spare * bs, case["hkv"] * case["d"]))
        self.dims = None

    def run(self, case):
        if own:
            from paper_2512_17910_amd import binding as ab
            if self.dims is None:
                self.dims = ab.make_cache_dims([y[0] for y in self.caches], [y[1] for y in self.caches], case["hkv"], case["d"], case["bs"])
            ab.alora_cache_move_rows(self.src, self.dst, self.shift if self.rope else None, self.rope, self.dims, interleaved=case["interleaved"])
            return self.caches
        k = self.caches[:, 0, self.src]
        if self.rope:
            c, s = (x[self.shift.abs().long()][:, None, :] for x in self.rope)
            s = torch.where((self.shift < 0)[:, None, None], -s, s)
            k = _plain_turn(k.float().view(case["layers"], case["rows"], case["hkv"], case["d"]), c, s, case).to(k.dtype).view(k.shape)
        self.caches[:, 0, self.dst] = k
        self.caches[:, 1, self.dst] = self.caches[:, 1, self.src]
        return self.caches


# ---- the plain forms ----------------------------------------------------------------------------
def _plain_turn(x, c, s, case):
    """fp32 heads, turned by the angles of cosines and sines `c`, `s`."""
    rot = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _plain_heads(x, w, c, s, case):
    y = x.float()
    if case["norm"]:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    if c is not None:
        y = _plain_turn(y, c, s, case)
    return y.to(x.dtype)


def _plain_heads_back(x, dy, w, c, s, case):
    g = _plain_turn(dy.float(), c, -s, case)
    if not case["norm"]:
        return g.to(x.dtype), None
    y = x.float()
    r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    u = g * w.float()
    dx = r * u - y * (r * r * r) * (u * y).mean(-1, keepdim=True)
    return dx.to(x.dtype), (g * y * r).sum((0, 1))


# ---- the definitions in 64 bits -----------------------------------------------------------------
def _exact_turn(x, pos, cos, sin, case):
    """The rotation as a product of complex numbers; `pos` gives each row's angles, the way back where it is negative."""
    rot = case["rot"]
    phase = torch.complex(cos.double()[pos.abs().long()], torch.sign(pos.double() + 0.5)[:, None] * sin.double()[pos.abs().long()])
    turned, rest = x[..., :rot], x[..., rot:]
    if case["interleaved"]:
        z = torch.view_as_complex(turned.reshape(*turned.shape[:-1], rot // 2, 2).contiguous()) * phase[:, None, :]
        turned = torch.view_as_real(z).reshape(turned.shape)
    else:
        z = torch.complex(turned[..., : rot // 2], turned[..., rot // 2:]) * phase[:, None, :]
        turned = torch.cat((z.real, z.imag), -1)
    return torch.cat((turned, rest), -1)


def _exact_heads(x, w, pos, rope, case):
    y = x
    if w is not None:
        y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["d"] + EPS) * w
    return _exact_turn(y, pos, *rope, case) if rope else y


def exact(case, seed):
    if case["kind"] == "blocks":
        st = _Blocks(case, seed)
        order = np.arange(case["blocks"])
        order[st.dst] = st.src
        out = st.caches.index_select(2, _dev(np.maximum(order, 0)))
        return out.masked_fill_(_dev(order < 0)[None, None, :, None], 0.0)
    if case["kind"] == "tables":
        st = _Tables(case, seed)
        i = np.arange(case["rot"] // 2, dtype=np.float64)
        theta = np.exp(-2.0 * i / case["rot"] * math.log(st.base))
        if case["scaling"] != "none":
            keep = 0.0 if case["scaling"] == "linear" else np.clip(
                (case["original"] * theta / (2.0 * math.pi) - case["low"]) / (case["high"] - case["low"]), 0.0, 1.0)
            theta = theta * keep + theta / case["factor"] * (1.0 - keep)
        z = case["magnitude"] * np.exp(1j * np.outer(np.arange(case["rows"], dtype=np.float64) + st.first, theta))
        return np.ascontiguousarray(z.real), np.ascontiguousarray(z.imag)
    if case["kind"] == "rows":
        st = _Rows(case, seed)
        out = st.caches.double() if case["rot"] else st.caches.clone()
        if case["rot"]:
            k = out[:, 0].index_select(1, st.src).view(case["layers"], case["rows"], case["hkv"], case["d"])
            k = _exact_turn(k, st.shift, *st.rope, case)
        else:
            k = out[:, 0].index_select(1, st.src)
        v = out[:, 1].index_select(1, st.src)
        out[:, 0].index_copy_(1, st.dst, k.view(v.shape))
        out[:, 1].index_copy_(1, st.dst, v)
        return out
    t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
    if case["kind"] == "heads":
        st = _Heads(case, seed)
        wq, wk = (None, None) if not case["norm"] else (st.wq.double(), st.wk.double())
        q = _exact_heads(st.q.double().view(t, hq, d), wq, st.pos, st.rope, case).view(t, hq * d)
        kc, vc, n = st.kc.double(), st.vc.double(), t - case["pad"]
        k = (kc.index_select(0, st.slot[:n]) if st.k is None else st.k.double()[:n]).view(n, hkv, d)
        kc.index_copy_(0, st.slot[:n], _exact_heads(k, wk, st.pos[:n], st.rope, case).reshape(n, hkv * d))
        if st.v is not None:
            vc.index_copy_(0, st.slot[:n], st.v.double()[:n])
        return q, kc, vc
    st = _HeadsBack(case, seed)         # differentiated: the definition above, its products with the outputs' gradients summed
    wq, wk = (None, None) if not case["norm"] else (w.double().requires_grad_() for w in (st.wq, st.wk))
    q, k = (x.double().view(t, -1, d).requires_grad_() for x in (st.q, st.k))
    total = (_exact_heads(q, wq, st.pos, st.rope, case) * st.dq_out.double().view(t, hq, d)).sum() + \
        (_exact_heads(k, wk, st.pos, st.rope, case) * st.dk_out.double().view(t, hkv, d)).sum()
    got = torch.autograd.grad(total, [q, k] + ([wq, wk] if case["norm"] else []))
    return got[0].reshape(t, hq * d), got[1].reshape(t, hkv * d), *(got[2:] or (None, None))


_KINDS = {"heads": _Heads, "heads-back": _HeadsBack, "tables": _Tables, "blocks": _Blocks, "rows": _Rows}


def prepare(case, seed):
    return case, _KINDS[case["kind"]](case, seed)


def run(state):
    case, st = state
    return st.run(case)


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    if case["kind"] == "tables":
        n = case["rows"] * (case["rot"] // 2)
        return {"bytes": 8.0 * n, "flops": 8.0 * n}
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "blocks":
        block = 2.0 * case["layers"] * case["bs"] * case["hkv"] * case["d"] * e
        return {"bytes": block * (2 * case["pairs"] - case["clears"]), "flops": 0.0}
    if case["kind"] == "rows":
        n = 2.0 * case["layers"] * case["rows"] * case["hkv"] * case["d"]
        return {"bytes": 2 * n * e + case["rows"] * (16 + (4 if case["rot"] else 0)), "flops": 3.0 * n / 2 * case["rot"] / case["d"]}
    t, hq, hkv, d = case["rows"], case["hq"], case["hkv"], case["d"]
    n = t * (hq + hkv) * d
    angles = 4.0 * t * case["rot"] + 4 * t                          # each row's cosines and sines, and its position
    if case["kind"] == "heads":
        copied = t * hkv * d if case["form"] == "buffer" else 0
        return {"bytes": 2.0 * e * (n + copied) + angles + 8 * t, "flops": n * ((4.0 if case["norm"] else 0.0) + 3.0 * case["rot"] / d)}
    return {"bytes": 3.0 * e * n + angles, "flops": n * ((11.0 if case["norm"] else 0.0) + 3.0 * case["rot"] / d)}
