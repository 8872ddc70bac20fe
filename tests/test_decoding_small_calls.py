"""Calls at the small end of what trees and selections allow, their launches found without a GPU (see launch_recorder.c)."""
import json
import os
import subprocess
import sys

import pytest

import test_decoding_abi as abi
import test_decoding_launches as launches

HERE = os.path.dirname(os.path.abspath(__file__))
ab = abi.ab
run_tree = launches.run_tree


def run_select(size, **kw):
    return abi.select(abi.attn(**kw), size=size)


def run_selected(size, budget, **kw):
    return abi.selected(abi.attn(**kw), budget=budget, size=size)


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    rec = str(tmp_path_factory.mktemp("rec") / "librec.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", "-o", rec, os.path.join(HERE, "launch_recorder.c")], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-c", launches.RECORD.replace("import test_decoding_launches", "import test_decoding_small_calls"), rec, HERE, os.path.dirname(HERE)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, (r.returncode, r.stderr[-3000:])
        return json.loads(r.stdout)
    return run


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("group", [1, 2, 4, 8])
def test_trees_of_no_sequences(recorder, dtype, head_dim, group):
    """A padded batch of which nothing is left, of fewer rows than a tile: they are cleared, and there is nothing to combine."""
    calls = [["run_tree", dict(dtype=dtype, head_dim=head_dim, n_q_heads=2 * group, n_seqs=0, n_tokens=n)] for n in (1, 2, 15, 16, 127, 128, 130)]
    for (status, found), (_, kw) in zip(recorder(calls), calls):
        assert status == ab.ALORA_OK and [l[0] for l in found][:1] == [f"tree_{'matrix' if dtype else 'vector'}_kernel"]
        assert all(x > 0 for _, _, grid, block in found for x in (*grid, *block)), kw


SERVERS = [dict(n_q_heads=32, n_kv_heads=8), dict(n_q_heads=8, n_kv_heads=1), dict(n_q_heads=5, n_kv_heads=5, dtype=0, head_dim=64), dict(n_q_heads=300, n_kv_heads=300),
           dict(n_q_heads=600, n_kv_heads=600)]
ROWS = (1, 2, 31, 32, 33, 63, 64, 65, 128, 129, 256, 300, 512, 700)


@pytest.mark.parametrize("heads", SERVERS, ids=lambda h: str(h["n_kv_heads"]))
def test_a_workspace_is_enough_for_fewer_rows(recorder, heads):
    """A server makes its buffer for its largest batch; every smaller one runs in it."""
    calls, sizes = [], []
    for columns, budget in ((100, 9), (900, 128), (4096, 128), (5000, 700)):
        d = [abi.attn(**heads, n_tokens=n, max_blocks=columns, n_seqs=n) for n in ROWS]
        for name, run, more, kw in (("alora_block_select", "run_select", (), {}), ("alora_selected_attention", "run_selected", (budget,), dict(budget=budget))):
            size = [abi.size_of(name, x, *more)[1] for x in d]
            assert size == sorted(size), (name, columns, size)
            at = ROWS.index(300)
            for n in sorted({*range(1, 300, 7), 31, 32, 63, 64, 65, 128, 256, 300}):
                calls.append([run, dict(heads, **kw, n_tokens=n, max_blocks=columns, n_seqs=n, size=size[at])])
    assert all(status == ab.ALORA_OK for status, _ in recorder(calls)), [c for (s, _), c in zip(recorder(calls), calls) if s][:3]
