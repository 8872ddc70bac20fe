"""Trees over tables that reach further than 2^29 positions (alora_tree.h)."""
import pytest
import torch

from paper_2512_17910_amd import binding as ab
from gpu_util import raw_bits
from test_gpu_decoding import Tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,n", [([5000, 20, 700], [13, 40, 64]), ([9000], [1]), ([1200] * 40 + [31, 0], [9] * 42)], ids=["few", "one", "many"])
@pytest.mark.parametrize("columns", [1 << 25, (1 << 25) + 1])          # of 16 positions: as many as parts count in units of 32, and of 64
def test_trees_over_large_tables(dtype, ctx, n, columns):
    t = Tree(dtype, ctx, n, 1, 16, 8, 64, 16, seed=21)
    wide = torch.full((len(n), columns), -1, dtype=torch.int32, device="cuda")
    wide[:, : t.bt.shape[1]] = t.bt
    t.bt = wide
    t.dims = ab.make_attn_dims(t.q, t.cache.k, wide, 16, 8, 64, 16)
    need = ab.alora_tree_attention_workspace_bytes(t.dims, 1) // 4
    t.ws = torch.full((need + 64,), 7.0, device="cuda")
    first = raw_bits(t.run()).copy()
    assert (t.ws[need:] == 7.0).all()
    t.check()
    t.ws.fill_(-1e30)
    t.out.fill_(float("nan"))
    assert (raw_bits(t.run()) == first).all()
