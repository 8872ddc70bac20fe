"""The launches of steps, trees and selections -- kernels, grids -- found without a GPU (see launch_recorder.c)."""
import itertools
import json
import os
import subprocess
import sys

import pytest

import test_decoding_abi as t
from paper_2512_17910_amd import binding as ab

HERE = os.path.dirname(os.path.abspath(__file__))
RECORD = """
import ctypes, json, re, sys, types
sys.modules["torch"] = types.ModuleType("torch")         # (the real one would register kernels of its own)
rec = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)      # ahead of the library: its HIP calls bind here
sys.path[:0] = sys.argv[2:4]
import test_decoding_launches as t
from launches import _Launch
t.ab._lib = t.ab.lib()
rec.rec_get.restype = ctypes.POINTER(_Launch)
out = []
for name, args in json.load(sys.stdin):
    rec.rec_reset()
    status = getattr(t, name)(**args)
    launches = []
    for i in range(rec.rec_count()):
        r = rec.rec_get(i).contents
        m = re.search(r"N5alora(\\d+)", r.name.decode())
        name = r.name.decode()[m.end():m.end() + int(m.group(1))]
        launches.append([name, [int(v) for v in re.findall(r"L[ib](\\d+)E", r.name.decode())], list(r.grid), list(r.block)])
    out.append([status, launches])
print(json.dumps(out))
"""


def run_step(**kw):
    return t.step(**kw)


def run_tree_rows(**kw):
    return t.tree_rows(**kw)


def run_tree(words=1, **kw):
    return t.tree(t.attn(**kw), words=words, size=1 << 60)


def run_select(**kw):
    return t.select(t.attn(**kw), size=1 << 60)


def run_selected(budget=9, **kw):
    return t.selected(t.attn(**kw), budget=budget, size=1 << 60)


def run_bounds(**kw):
    import ctypes
    d = ab.AloraBoundsDims(**{**dict(dtype=1, n_rows=5, n_kv_heads=2, head_dim=64, block_size=16, n_slots=160), **kw})
    return ab.lib().alora_block_bounds(t.P, t.P, t.P, t.P, ctypes.byref(d), None)


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    rec = str(tmp_path_factory.mktemp("rec") / "librec.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", "-o", rec, os.path.join(HERE, "launch_recorder.c")], check=True)

    def run(*calls):
        r = subprocess.run([sys.executable, "-c", RECORD, rec, HERE, os.path.dirname(HERE)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-3000:]
        out = json.loads(r.stdout)
        for (status, launches), call in zip(out, calls):
            assert status == ab.ALORA_OK, call
            for _, _, grid, block in launches:
                assert all(0 < g * b < 1 << 32 for g, b in zip(grid, block)) and grid[1] < 65536 and grid[2] < 65536, (call, launches)
        return [launches for _, launches in out]
    return run


def test_steps_and_tree_rows(record):
    one, rows, pool, most = record(["run_step", {}], ["run_step", dict(row_cap=5000)], ["run_step", dict(pool_cap=40000)], ["run_step", dict(row_cap=1 << 30, pool_cap=1 << 30)])
    assert [l[0][2] for l in (one, rows, pool, most)] == [[1, 1, 1], [39, 1, 1], [39, 1, 1], [1024, 1, 1]] and one[0][0] == "step_rows_kernel" and len(one) == 1
    for words in (1, 2, 3, 4):
        few, many = record(["run_tree_rows", dict(words=words)], ["run_tree_rows", dict(words=words, tokens=2**31 - 1, seqs=1 << 20)])
        assert few == [["tree_rows_kernel", [words], [3, 1, 1], [64 * words, 1, 1]]] and many[0][2] == [(1 << 20) + 64, 1, 1]


def test_trees(record):
    """Rows of a tile by type and group; which kernel by the rows that a sequence brings on average."""
    wide = dict(n_q_heads=32, n_kv_heads=8, n_seqs=5)
    calls = [(16, "tree_matrix_kernel", [128, 1, 1]), (17, "tree_matrix_kernel", [128, 1, 0]), (32, "tree_matrix_kernel", [128, 1, 0]), (33, "tree_matrix_kernel", [128, 0, 0])]
    for (rows, name, ints), launches in zip(calls, record(*[["run_tree", dict(wide, n_tokens=5 * n)] for n, _, _ in calls])):
        items = 5 * rows // 32 + 5 + 2 * 64 + 2
        assert launches == [[name, ints, [(items + 1 + 5 * rows // 64) * 8, 1, 1], [256, 1, 1]], ["tree_merge_kernel", [128, 1, 8], [(5 * rows // 32 + 5) * 8, 32, 1], [256, 1, 1]]]
    plans = [(64, []), (65, [["tree_plan_kernel", [256], [1, 1, 1], [256, 1, 1]]]), (512, [["tree_plan_kernel", [256], [1, 1, 1], [256, 1, 1]]]),
             (513, [["tree_plan_kernel", [1024], [1, 1, 1], [1024, 1, 1]]])]
    for (seqs, plan), launches in zip(plans, record(*[["run_tree", dict(wide, n_tokens=8 * n, n_seqs=n)] for n, _ in plans])):
        tiles = seqs // 4 + seqs
        assert launches[:-2] == plan and launches[-1][2] == [8 * tiles, max(1, min(32, 8192 // (8 * tiles))), 1]
    for g, columns in ((1, 4), (2, 4), (4, 4), (8, 8)):
        l, = record(["run_tree", dict(dtype=0, n_q_heads=2 * g, n_tokens=40)])
        assert l[0][1] == [128, columns] and l[0][2][0] == 2 * (40 * g // columns + 2 + 512 + 2 + 1) and l[1][1] == [128, 0, 8]
    assert record(["run_tree", dict(n_tokens=0)]) == [[]]
    record(["run_tree", dict(n_tokens=1 << 22, words=4)], ["run_tree", dict(n_tokens=1 << 21, dtype=0, n_q_heads=16)])     # (large ones fit a grid)


def test_selections(record):
    one = dict(n_kv_heads=8, n_q_heads=32, n_tokens=3, max_blocks=512, n_seqs=3)
    few, far, many, wide, chunk = record(["run_select", one], ["run_select", dict(one, max_blocks=513)], ["run_select", dict(one, max_blocks=4352, n_tokens=32)],
                                         ["run_select", dict(one, max_blocks=4353, n_tokens=70000)], ["run_select", dict(one, n_tokens=200, n_seqs=9)])
    assert few == [["block_select_kernel", [128, 1, 1], [24, 1, 1], [256, 1, 1]]] and many[0][:3] == ["block_select_kernel", [128, 1, 0], [256, 1, 1]]
    assert far == [["block_keys_kernel", [128, 1, 1], [9, 3, 2], [256, 1, 1]], ["block_list_kernel", [1024], [24, 1, 1], [1024, 1, 1]]]
    assert [l[0] for l in wide] == ["block_keys_kernel", "block_keys_kernel", "block_list_kernel"] and [l[2] for l in wide] == [[69, 65535, 2], [69, 4465, 2], [560000, 1, 1]]
    assert chunk[0][:2] == ["block_select_kernel", [128, 1, 0]]
    record(["run_select", dict(n_tokens=(1 << 21) - 1, max_blocks=1 << 28)], ["run_select", dict(n_tokens=63, n_kv_heads=1 << 16, n_q_heads=1 << 16, max_blocks=5000)])


def test_selected_lists_fill_the_chip(record):
    """512 lists, or a multiple, are read whole; others behind them in parts while that is faster."""
    one = dict(n_kv_heads=8, n_q_heads=32)
    for rows, budget in itertools.product((1, 7, 64, 65, 200, 256, 1000), (1, 4, 33, 128, 4000)):
        l, = record(["run_selected", dict(one, n_tokens=rows, budget=budget)])
        lists, rest = rows * 8, rows * 8 % 512
        if len(l) == 1:
            assert l[0][2][0] == lists and (rest == 0 or budget <= 33)
        else:
            parts, left = divmod(l[0][2][0] - (lists - rest), rest)
            assert left == 0 and 2 <= parts <= 32 and l[1][0] == "selected_merge_kernel" and l[1][2] == [rest, 1, 1]
    assert record(["run_selected", dict(one, n_tokens=1, budget=128)])[0][0][2][0] >= 8 * 16


def test_bounds(record):
    small, some, large, most = record(*[["run_bounds", dict(n_rows=n)] for n in (1024, 1025, 4097, 1 << 27)])
    assert some == [["block_bounds_kernel", [64, 1, 4], [257, 1, 1], [256, 1, 1]]]
    assert small == [["block_bounds_kernel", [64, 1, 2], [512, 1, 1], [256, 1, 1]]] and large == [["block_bounds_kernel", [64, 1, 16], [257, 1, 1], [256, 1, 1]]]
    assert most[0][2] == [1 << 23, 1, 1]


def test_every_instantiation_is_reached(record):
    """By calls of the sizes that the tests on the GPU run."""
    calls = []
    for dtype, d, g in itertools.product((0, 1), (64, 128), (1, 2, 4, 8)):
        shape = dict(dtype=dtype, head_dim=d, n_q_heads=2 * g, n_seqs=6)
        calls += [["run_tree", dict(shape, n_tokens=6 * n // g)] for n in (30, 100, 300)] + [["run_tree", dict(shape, n_tokens=3, n_seqs=n)] for n in (1, 300, 600)]
        calls += [["run_select", dict(shape, n_tokens=n, max_blocks=m)] for n in (6, 40) for m in (100, 900)] + [["run_selected", dict(shape, n_tokens=n, budget=40)] for n in (6, 40)]
        calls += [["run_bounds", dict(dtype=dtype, head_dim=d, n_rows=n)] for n in (60, 1300, 4600)]
    calls += [["run_step", {}]] + [["run_tree_rows", dict(words=w)] for w in (1, 2, 3, 4)]
    reached = {(name, *ints) for launches in record(*calls) for name, ints, _, _ in launches}
    D, B = (64, 128), (0, 1)
    want = {("step_rows_kernel",), ("tree_plan_kernel", 256), ("tree_plan_kernel", 1024), ("block_list_kernel", 1024), *(("tree_rows_kernel", w) for w in (1, 2, 3, 4))}
    for d in D:
        want |= {("tree_vector_kernel", d, c) for c in (4, 8)} | {("tree_matrix_kernel", d, *x) for x in ((1, 1), (1, 0), (0, 0))}
        want |= {("selected_vector_kernel", d, g) for g in (1, 2, 4, 8)} | {("selected_matrix_kernel", d, once) for once in B}
        for b in B:
            want |= {("tree_merge_kernel", d, b, 8), ("tree_merge_kernel", d, 1, 16), ("selected_merge_kernel", d, b)} | {("block_bounds_kernel", d, b, n) for n in (2, 4, 16)}
            want |= {(k, d, b, once) for k in ("block_select_kernel", "block_keys_kernel") for once in B}
    assert reached == want
    # ... and the library holds no others of them
    text = open(ab.LIB_PATH, "rb").read()
    import re
    names = {m.group(0).decode() for m in re.finditer(rb"_ZN5alora\d+(step_rows|tree_\w+?|block_(?:bounds|select|keys|list)|selected_\w+?)_kernel[A-Za-z0-9_]*", text)}
    def parsed(n):
        m = re.search(r"N5alora(\d+)", n)
        return (n[m.end():m.end() + int(m.group(1))], *[int(v) for v in re.findall(r"L[ib](\d+)E", n)])
    assert {parsed(n) for n in names} == want
