"""Calls at the small end of what trees and selections allow (alora_tree.h, alora_select.h)."""
import pytest
import torch

from paper_2512_17910_amd import binding as ab
from test_gpu_decoding import DT, Select

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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_workspace_for_batches_of_any_size(dtype):
    """Made for 70 rows, used for fewer: lists and attention as in a workspace of their own."""
    s = Select(dtype, [800 + 9 * i for i in range(70)], 8, 8, 64, 1, seed=1)
    hq, hkv, d = s.sizes
    new = lambda n: torch.empty((n,), dtype=torch.uint8, device="cuda")
    big = [new(ab.alora_block_select_workspace_bytes(s.dims)), new(ab.alora_selected_attention_workspace_bytes(s.dims, 40))]
    for n in (70, 64, 63, 32, 31, 1):
        q, rows = s.q[:n], [x[:n].contiguous() for x in s.dev]
        dims = ab.make_attn_dims(q, s.cache.k, s.bt, hq, hkv, d, 1)
        got = []
        for ws in (big, [new(ab.alora_block_select_workspace_bytes(dims)), new(ab.alora_selected_attention_workspace_bytes(dims, 40))]):
            sel, out = torch.full((n, hkv, 40), -9, dtype=torch.int32, device="cuda"), torch.full_like(q, NAN)
            ab.alora_block_select(q, s.b, s.s, s.bt, *rows, sel, 1, 2, dims, ws[0])
            ab.alora_selected_attention(q, s.cache.k, s.cache.v, s.bt, *rows, sel, out, dims, ws[1])
            got.append((sel, out))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and torch.isfinite(got[0][1]).all(), n
