"""One layer's attention inside the example (paper_2512_17910_amd/speculation.py), where no layer behind it spreads a difference."""
import pytest

from paper_2512_17910_amd import speculation
from gpu_util import TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_size", [16, 5])
def test_all_blocks_selected_are_the_whole_context(dtype, block_size):
    """Of the same queries and cache: each reader's own gate."""
    r = speculation.run(layers=2, prompt=150, dtype=dtype, answer=6, block_size=block_size)
    print(r, flush=True)
    assert r["all_blocks_attention_off"] <= 2 * TOL[dtype] and r["some_blocks_finite"]
