"""Fork, compact and drop of the planner (include/alora_planner.h) on a simulated cache: what the planner says is done with the
contents of slots, and every live request has to find in its blocks what belongs there.  Host code only.

A row's content is named by all that its key and value depend on: the tokens up to it, where its adapter was active, and, for rows
that a drop moved, where they came from and by how much they were shifted.  Rows behind a drop see contents of their own and have
names that no other request may find."""
import ctypes
import os
import random
import subprocess
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
if __name__ == "__main__":
    sys.path[:0] = [ROOT, HERE]

from paper_2512_17910_amd import planner as pl  # noqa: E402
from paper_2512_17910_amd.binding import ALORA_EINVAL, ALORA_ESHAPE, AloraError  # noqa: E402

NEVER = 1 << 30


class Sim:
    def __init__(self, bs, n_blocks):
        self.p, self.bs, self.n_blocks = pl.Planner(bs, n_blocks), bs, n_blocks
        self.cache, self.reqs, self.names = {}, {}, 0

    def close(self):
        self.p.close()

    def _rows(self, r, first):
        for pos in range(first, len(r["tokens"])):
            if r["private"]:
                self.names += 1
                r["rows"].append(("private", self.names))
            else:
                active = r["adapter"] >= 0 and pos >= r["start"]
                r["rows"].append((tuple(r["tokens"][: pos + 1]), (r["adapter"], r["start"]) if active else None))

    def _project(self, rid, batch, first):
        r, (pos, seg, aid, slot, start) = self.reqs[rid], batch.rows()
        self._rows(r, first)
        assert list(pos) == list(range(first, len(r["tokens"]))) and list(start) == [r["start"]] and set(aid) <= {r["adapter"]}
        for p, s in zip(pos, slot):
            assert 0 <= s < self.n_blocks * self.bs
            self.cache[int(s)] = r["rows"][p]

    def admit(self, rid, tokens, adapter, start):
        b = pl.Batch(len(tokens), 1)
        cached = self.p.admit(rid, tokens, adapter, start, b)
        self.reqs[rid] = r = dict(tokens=list(tokens), adapter=adapter, start=start, rows=[], private=False)
        self._rows(r, 0)
        r["rows"] = r["rows"][:cached]
        self._project(rid, b, cached)
        return cached

    def append(self, rid, tokens):
        b, r = pl.Batch(len(tokens), 1), self.reqs[rid]
        first = len(r["tokens"])
        self.p.append(rid, tokens, b)
        r["tokens"] += list(tokens)
        self._project(rid, b, first)

    def commit(self, rid):
        self.p.commit(rid)

    def finish(self, rid):
        self.p.finish(rid)
        del self.reqs[rid]

    def _copy(self, src, dst):
        assert len(set(dst)) == len(dst) and not set(dst) & set(src)           # what alora_cache_copy_blocks takes
        for s, d in zip(src.tolist(), dst.tolist()):
            assert 0 <= s < self.n_blocks and 0 <= d < self.n_blocks
            for o in range(self.bs):
                self.cache[d * self.bs + o] = self.cache.get(s * self.bs + o)

    def fork(self, rid, new, adapter, start):
        src, dst = self.p.fork(rid, new, adapter, start)
        assert len(src) == (1 if len(self.reqs[rid]["tokens"]) % self.bs else 0)
        self._copy(src, dst)
        r = self.reqs[rid]
        self.reqs[new] = dict(r, tokens=list(r["tokens"]), rows=list(r["rows"]), adapter=adapter, start=start)

    def compact(self, n_blocks):
        src, dst = self.p.compact(n_blocks)
        assert (dst < n_blocks).all() and (src >= n_blocks).all()
        self._copy(src, dst)
        self.n_blocks = n_blocks
        for s in [s for s in self.cache if s >= n_blocks * self.bs]:
            del self.cache[s]

    def drop(self, rid, first, n):
        src, dst, shift = self.p.drop(rid, first, n)
        assert len(set(dst)) == len(dst) and not set(dst) & set(src) and ((shift == 0) | (shift == -n)).all()
        r = self.reqs[rid]
        moved = [(self.cache.get(int(s)), int(h)) for s, h in zip(src, shift)]
        for d, (content, h) in zip(dst.tolist(), moved):
            self.cache[d] = (content, h) if h else content
        behind = r["rows"][first + n:]
        r["rows"] = r["rows"][:first] + [(c, -n) for c in behind]
        del r["tokens"][first: first + n]
        if r["start"] >= first + n:
            r["start"] -= n
        elif r["start"] > first:
            r["start"] = first
        r["private"] = True

    def check(self):
        used = {}
        for rid, r in self.reqs.items():
            table = self.p.block_table(rid)
            assert len(table) == -(-len(r["tokens"]) // self.bs)
            for pos, content in enumerate(r["rows"]):
                assert self.cache.get(int(table[pos // self.bs]) * self.bs + pos % self.bs) == content, (rid, pos)
            for i, b in enumerate(table):
                used.setdefault(int(b), []).append((rid, i))
            assert ((0 <= table) & (table < self.n_blocks)).all()
        for b, holders in used.items():       # a block of several requests is full in all of them
            if len(holders) > 1:
                for rid, i in holders:
                    assert (i + 1) * self.bs <= len(self.reqs[rid]["tokens"])
        assert self.p.free_blocks() == self.n_blocks - len(used)


def test_fork_shares_full_blocks_and_copies_the_partial_one():
    s = Sim(4, 10)
    s.admit(1, list(range(10)), -1, NEVER)
    s.fork(1, 2, 7, 10)
    t1, t2 = s.p.block_table(1), s.p.block_table(2)
    assert list(t1[:2]) == list(t2[:2]) and t1[2] != t2[2] and s.p.free_blocks() == 6
    s.append(1, [90, 91, 92])
    s.append(2, [80, 81, 82])
    s.check()
    s.commit(1)
    s.commit(2)
    # the shared blocks are the base model's, the adapter's own block is not
    assert s.admit(3, list(range(10)) + [90, 91, 92], -1, NEVER) == 12 and s.admit(4, list(range(8)) + [1, 2], 3, 9) == 8
    s.check()
    s.finish(1)
    s.check()
    s.fork(2, 5, 7, 10)                       # an answer sampled twice: the adapter is active in both
    s.append(5, [1])
    s.check()
    s.close()


def test_fork_of_a_full_last_block_copies_nothing():
    s = Sim(4, 2)
    s.admit(1, list(range(8)), -1, NEVER)
    s.fork(1, 2, 0, 8)
    assert s.p.free_blocks() == 0
    s.check()
    with pytest.raises(AloraError) as e:
        s.append(2, [1])
    assert e.value.status == pl.ALORA_ENOBLOCKS
    s.close()


def test_forks_that_are_refused():
    s = Sim(4, 4)
    s.admit(1, list(range(6)), 3, 4)
    for new, adapter, start, status in ((1, 3, 4, ALORA_EINVAL), (2, -1, 0, ALORA_EINVAL), (2, 3, 5, ALORA_EINVAL), (2, 4, 4, ALORA_EINVAL),
                                        (2, 4, 6, ALORA_EINVAL), (2, -2, 4, ALORA_EINVAL), (2, 3, -1, ALORA_EINVAL)):
        with pytest.raises(AloraError) as e:
            s.p.fork(1, new, adapter, start)
        assert e.value.status == status, (new, adapter, start)
    with pytest.raises(AloraError):
        s.p.fork(9, 2, 3, 4)
    s.admit(5, list(range(100, 108)), -1, NEVER)
    with pytest.raises(AloraError) as e:
        s.p.fork(5, 6, 2, 7)                  # active at position 7, which the base model projected
    assert e.value.status == ALORA_EINVAL
    with pytest.raises(AloraError) as e:
        s.p.fork(1, 2, 3, 4)                  # no block for the partial one
    assert e.value.status == pl.ALORA_ENOBLOCKS
    s.check()
    s.close()


def test_compact_moves_what_is_used_and_keeps_what_is_reusable():
    s = Sim(4, 12)
    for i in range(5):
        s.admit(i, [10 * i + j for j in range(8)], -1, NEVER)     # blocks 0 .. 9
        s.commit(i)
    for i in (0, 2):
        s.finish(i)
    assert s.admit(7, list(range(8)) + [1], -1, NEVER) == 8       # blocks 0, 1 again, and 10
    with pytest.raises(AloraError) as e:
        s.p.compact(8)
    assert e.value.status == pl.ALORA_ENOBLOCKS
    s.check()
    s.compact(9)
    s.check()
    assert s.p.free_blocks() == 0
    s.finish(4)
    assert s.admit(8, [40 + j for j in range(8)], -1, NEVER) == 4  # reused from where its blocks went
    s.check()
    s.close()


def test_compact_arguments():
    p = pl.Planner(4, 6)
    L, n = pl._L(), ctypes.c_int32(9)
    a = np.zeros(6, np.int32)
    assert L.alora_planner_compact(None, 3, a.ctypes.data, a.ctypes.data, 6, ctypes.byref(n)) == ALORA_EINVAL
    for blocks, src, cap in ((-1, a.ctypes.data, 6), (7, a.ctypes.data, 6), (3, None, 1), (3, a.ctypes.data, -1)):
        assert L.alora_planner_compact(p._h, blocks, src, a.ctypes.data, cap, ctypes.byref(n)) == ALORA_EINVAL
    b = pl.Batch(24, 3)
    for i in range(3):
        p.admit(i, list(range(8 * i, 8 * i + 8)), -1, NEVER, b)
    for i in (0, 1):
        p.finish(i)
    assert L.alora_planner_compact(p._h, 3, a.ctypes.data, a.ctypes.data, 1, ctypes.byref(n)) == ALORA_ESHAPE and n.value == 2
    assert p.free_blocks() == 4 and not a.any()
    src, dst = p.compact(2)
    assert sorted(src) == [4, 5] and sorted(dst) == [0, 1] and p.free_blocks() == 0
    src, dst = p.compact(2)
    assert len(src) == len(dst) == 0


def test_drop():
    s = Sim(4, 24)
    s.admit(1, list(range(18)), 2, 9)
    s.commit(1)
    s.fork(1, 2, 2, 9)
    s.drop(1, 5, 6)                           # the activation point is among them
    assert s.reqs[1]["start"] == 5 and s.reqs[1]["tokens"] == list(range(5)) + list(range(11, 18))
    s.check()
    s.append(1, [70, 71, 72, 73, 74])
    s.check()
    s.commit(1)                               # only its first block is what its tokens say
    assert s.admit(3, list(range(5)) + list(range(11, 16)), 2, 5) == 4
    s.finish(2)
    assert s.admit(4, list(range(18)), 2, 9) == 16               # the old blocks are reusable still
    s.check()
    s.finish(3)
    s.drop(1, 0, 3)
    s.check()
    s.drop(1, 12, 2)                          # the last tokens, at a border: nothing moves
    s.check()
    for first, n in ((0, 12), (12, 1), (-1, 2), (3, 0), (5, 1 << 30)):
        with pytest.raises(AloraError) as e:
            s.p.drop(1, first, n)
        assert e.value.status == ALORA_EINVAL
    with pytest.raises(AloraError):
        s.p.drop(99, 0, 1)
    s.check()
    s.close()


def test_drop_needs_blocks():
    s = Sim(4, 4)
    s.admit(1, list(range(14)), -1, NEVER)
    with pytest.raises(AloraError) as e:
        s.drop(1, 0, 1)
    assert e.value.status == pl.ALORA_ENOBLOCKS
    s.check()
    s.close()


@pytest.mark.parametrize("seed", range(30))
def test_random_conversations(seed):
    rng = random.Random(seed)
    s = Sim(rng.choice([1, 2, 4, 5]), rng.choice([12, 30, 60]))
    done, next_id = {}, 0
    for _ in range(120):
        live = list(s.reqs)
        op = rng.choice(["admit", "admit", "append", "append", "commit", "commit", "finish", "fork", "fork", "compact", "drop", "drop"])
        try:
            if op == "admit" and len(live) < 6:
                next_id += 1
                n = rng.randint(1, 14)
                adapter = rng.choice([-1, -1, 0, 1])
                s.admit(next_id, [rng.choice([0, 0, 0, 1]) for _ in range(n)], adapter, NEVER if adapter < 0 else rng.randint(0, n + 2))
            elif not live:
                continue
            elif op == "append":
                s.append(rng.choice(live), [rng.choice([0, 1]) for _ in range(rng.randint(1, 7))])
            elif op == "commit":
                s.commit(rng.choice(live))
            elif op == "finish" and len(live) > 2:
                s.finish(rng.choice(live))
            elif op == "fork":
                next_id += 1
                rid = rng.choice(live)
                r = s.reqs[rid]
                same = rng.random() < 0.4
                s.fork(rid, next_id, r["adapter"] if same else rng.choice([-1, 0, 1]), r["start"] if same else rng.randint(len(r["tokens"]), len(r["tokens"]) + 2))
            elif op == "compact" and rng.random() < 0.3:
                s.compact(max(8, s.n_blocks - rng.randint(0, 6)) if s.n_blocks > 8 else s.n_blocks)
            elif op == "drop":
                rid = rng.choice(live)
                n = len(s.reqs[rid]["tokens"])
                if n > 1:
                    k = rng.randint(1, n - 1)
                    s.drop(rid, rng.randint(0, n - k), k)
        except AloraError as e:
            assert e.status in (pl.ALORA_ENOBLOCKS, ALORA_EINVAL) and (op == "fork" or e.status == pl.ALORA_ENOBLOCKS)
        done[op] = done.get(op, 0) + 1
        s.check()
    s.close()


@pytest.mark.parametrize("seed", [59, 272, 402, 419])
def test_random_conversations_whose_activation_points_share_a_block(seed):
    test_random_conversations(seed)


def test_a_fork_is_not_found_by_a_request_activated_elsewhere():
    s = Sim(4, 20)
    s.admit(1, list(range(10)), -1, NEVER)
    s.fork(1, 2, 0, 10)
    s.append(2, [10, 11, 12])
    s.commit(2)
    assert s.admit(3, list(range(13)), 0, 9) == 8        # position 9 of request 2 was projected by the base model
    s.check()
    assert s.admit(4, list(range(13)), 0, 10) == 12
    s.check()
    s.close()


def test_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    """The tests above on a build of the planner's host code with CPU sanitizers."""
    so = str(tmp_path / "planner_san.so")
    subprocess.run(["g++", "-x", "c++", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1",
                    "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-o", so,
                    os.path.join(ROOT, "paper_2512_17910_amd", "csrc", "alora_planner.hip")], check=True)
    asan = subprocess.run(["gcc", "-print-file-name=libasan.so"], check=True, capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    env["LD_PRELOAD"] = ":".join(p for p in (asan, env.get("LD_PRELOAD", "")) if p)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], env=env, capture_output=True, text=True, timeout=600)
    tail = r.stdout[-3000:] + "\n" + r.stderr[-3000:]
    assert r.returncode == 0 and "passed" in r.stdout and "ERROR: AddressSanitizer" not in tail and "runtime error" not in tail, tail


if __name__ == "__main__":
    pl.use_planner_library(ctypes.CDLL(sys.argv[1]))
    sys.exit(int(pytest.main(["-x", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__), "-k", "not sanitizers"])))
