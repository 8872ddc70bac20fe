"""Calls at the small end of what trees and selections allow, their launches found without a GPU (see launch_recorder.c)."""
import json
import os
import subprocess
import sys

import pytest

import test_decoding_launches as launches
from paper_2512_17910_amd import binding as ab

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    rec = str(tmp_path_factory.mktemp("rec") / "librec.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", "-o", rec, os.path.join(HERE, "launch_recorder.c")], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-c", launches.RECORD, rec, HERE, os.path.dirname(HERE)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
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
