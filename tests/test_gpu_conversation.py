"""The operators together, as they are used (paper_2512_17910_amd/conversation.py)."""
import pytest

from paper_2512_17910_amd import conversation
from gpu_util import TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(prompt=203), dict(prompt=100, interleaved=True, rotary_dim=64), dict(prompt=131, block_size=12, rotary_dim=20, layers=3)],
                         ids=["halves", "neighbours", "part"])
def test_conversation(dtype, kw):
    """Bounds: the gates of the projection and the reader, three calls a layer; the re-turned keys of the first layer one gate (two
    roundings instead of one, well inside)."""
    layers = kw.pop("layers", 2)
    r = conversation.run(layers=layers, dtype=dtype, **kw)
    print(r, flush=True)
    gate = TOL[dtype]
    assert r["fork_off"] <= 3 * layers * gate and r["forked_blocks_shared"] == (kw["prompt"] + 3) // kw.get("block_size", 16)
    assert r["moved_rows"] > 0 and r["drop_key_off"] <= gate and r["drop_value_off"] <= gate
    assert r["compacted_blocks"] > 0 and r["blocks"] < r["blocks_before"] and r["same_answer"]
    assert all(b < 0.5 * a for a, b in zip(r["loss"], r["loss"][1:])), r["loss"]
