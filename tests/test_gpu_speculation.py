"""Steps, trees and selections together, as they are used (paper_2512_17910_amd/speculation.py)."""
import pytest

from paper_2512_17910_amd import speculation
from gpu_util import TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(prompt=203, answer=12), dict(prompt=300, answer=30, block_size=5, seqs=4), dict(prompt=90, answer=8, layers=3)], ids=["plain", "odd-blocks", "deep"])
def test_speculation(dtype, kw):
    """Bounds: the gates of the projection, the heads and the reader, three calls a layer, of each side."""
    layers = kw.pop("layers", 2)
    r = speculation.run(layers=layers, dtype=dtype, **kw)
    print(r, flush=True)
    gate = 3 * layers * TOL[dtype]
    assert r["tokens"] > r["steps"] * kw.get("seqs", 3) and r["lengths"] and r["blocks_kept"]      # (some drafts were right)
    if dtype == "f32":
        assert r["same_as_told"] == r["told"]
    assert r["choice_gap"] <= 2 * gate and r["key_off"] <= gate and r["value_off"] <= gate
    assert r["all_blocks_off"] <= 2 * gate and r["some_blocks"] < r["of_blocks"]
