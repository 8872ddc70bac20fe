"""Calls of trees at the small end of what they allow (alora_tree.h)."""
import pytest
import torch

from paper_2512_17910_amd import binding as ab
from test_gpu_decoding import DT

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 3])
def test_a_few_rows_of_no_sequence(dtype, rows):
    """Fewer than a tile holds: zeros."""
    q, kv = torch.ones((rows, 512), device="cuda").to(DT[dtype]), torch.full((32, 128), NAN, device="cuda").to(DT[dtype])
    bt = torch.zeros((0, 4), dtype=torch.int32, device="cuda")
    dims = ab.make_attn_dims(q, kv, bt, 8, 2, 64, 16)
    none = torch.zeros((1,), dtype=torch.int32, device="cuda")
    mask, out = torch.full((rows, 1), -1, dtype=torch.int64, device="cuda"), torch.full_like(q, NAN)
    ws = torch.empty((ab.alora_tree_attention_workspace_bytes(dims, 1) + 16,), dtype=torch.uint8, device="cuda")
    ab.alora_tree_attention(q, kv, kv, bt, none, none[:0], mask, out, dims, ws)
    assert not out.any()
