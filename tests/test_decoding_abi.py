"""Refusals of steps, trees and selections, found on the host before anything is launched (CPU; dummy addresses that nothing dereferences)."""
import ctypes

import pytest
import torch

from paper_2512_17910_amd import binding as ab

P = 0x100000
OK, EINVAL, ESHAPE, EWORKSPACE = ab.ALORA_OK, ab.ALORA_EINVAL, ab.ALORA_ESHAPE, ab.ALORA_EWORKSPACE

STEP = ("lengths", "change", "kept", "adapters", "tables", "pool", "state", "lengths_out", "state_out", "offsets", "seq", "pos", "aid", "slot")


def step(kw=(), **d):
    dims = ab.AloraStepDims(**{**dict(n_seqs=3, max_blocks=4, block_size=16, row_cap=9, pool_cap=7, n_slots=160), **d})
    a = {n: P + 0x1000 * i for i, n in enumerate(STEP)}
    a.update(kw)
    return ab.lib().alora_step_rows(*[a[n] for n in STEP], ctypes.byref(dims), None)


def test_steps_are_refused():
    for kw, status in ((dict(n_seqs=-1), EINVAL), (dict(max_blocks=-1), EINVAL), (dict(block_size=0), EINVAL), (dict(row_cap=-1), EINVAL), (dict(pool_cap=-1), EINVAL),
                       (dict(n_slots=-1), EINVAL), (dict(n_seqs=(1 << 20) + 1), ESHAPE), (dict(row_cap=(1 << 30) + 1), ESHAPE), (dict(pool_cap=(1 << 30) + 1), ESHAPE),
                       (dict(n_slots=1 << 40, block_size=16), ESHAPE)):
        assert step(**kw) == status, kw
    for name in STEP:
        if name not in ("kept", "adapters"):
            assert step({name: None}) == EINVAL, name
        assert step({name: P + (4 if name == "slot" else 2)}) == EINVAL, name
    a = {n: P + 0x1000 * i for i, n in enumerate(STEP)}
    assert step({"lengths_out": a["lengths"]}) == step({"lengths_out": a["change"]}) == step({"state_out": a["state"]}) == EINVAL
    assert ab.lib().alora_step_rows(*[P] * 14, None, None) == EINVAL


def tree_rows(tokens=5, seqs=2, words=1, **kw):
    a = dict(parents=P, offsets=P, context=P, mask=P, pos=P)
    a.update(kw)
    return ab.lib().alora_tree_rows(a["parents"], a["offsets"], a["context"], a["mask"], a["pos"], tokens, seqs, words, None)


def test_tree_rows_are_refused():
    assert tree_rows(tokens=-1) == tree_rows(seqs=-1) == EINVAL
    assert tree_rows(words=0) == tree_rows(words=5) == tree_rows(seqs=(1 << 20) + 1) == ESHAPE
    for name in ("parents", "offsets", "context", "mask", "pos"):
        assert tree_rows(**{name: None}) == tree_rows(**{name: P + (4 if name == "mask" else 2)}) == EINVAL, name
    assert tree_rows(tokens=0, parents=None) == OK


def attn(**kw):
    return ab.AloraAttnDims(**{**dict(dtype=1, n_tokens=8, n_q_heads=8, n_kv_heads=2, head_dim=128, n_seqs=2, max_blocks=4, block_size=16, n_slots=128, scale=0.0), **kw})


SHAPES = [(dict(head_dim=96), ESHAPE), (dict(n_q_heads=6), ESHAPE), (dict(n_q_heads=7), ESHAPE), (dict(block_size=0), EINVAL), (dict(dtype=5), EINVAL),
          (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(n_tokens=-1), EINVAL), (dict(n_slots=1 << 31), ESHAPE)]
TREE = ("q", "k", "v", "tables", "offsets", "context", "mask", "out")
SELECT = ("q", "bounds", "scales", "tables", "seq", "pos", "selected")
SELECTED = ("q", "k", "v", "tables", "seq", "pos", "selected", "out")


def size_of(entry, d, *more):
    n = ctypes.c_size_t(0)
    s = getattr(ab.lib(), entry + "_workspace_bytes")(ctypes.byref(d), *more, ctypes.byref(n))
    return s, n.value


def tree(d, words=1, ws=P, size=1 << 40, **kw):
    a = {**{n: P for n in TREE}, **kw}
    return ab.lib().alora_tree_attention(*[a[n] for n in TREE[:7]], words, a["out"], ctypes.byref(d), ws, size, None)


def select(d, budget=9, first=1, recent=2, ws=P, size=1 << 40, **kw):
    a = {**{n: P for n in SELECT}, **kw}
    return ab.lib().alora_block_select(*[a[n] for n in SELECT], budget, first, recent, ctypes.byref(d), ws, size, None)


def selected(d, budget=9, ws=P, size=1 << 40, **kw):
    a = {**{n: P for n in SELECTED}, **kw}
    return ab.lib().alora_selected_attention(*[a[n] for n in SELECTED[:7]], budget, a["out"], ctypes.byref(d), ws, size, None)


@pytest.mark.parametrize("kw,status", SHAPES)
def test_readers_refuse_shapes(kw, status):
    d = attn(**kw)
    assert tree(d) == select(d) == selected(d) == status
    assert size_of("alora_tree_attention", d, 1)[0] == size_of("alora_block_select", d)[0] == size_of("alora_selected_attention", d, 9)[0] == status


def test_readers_refuse_arguments():
    d = attn()
    for call, names, loose in ((tree, TREE, ("tables", "offsets", "context")), (select, SELECT, ("scales", "tables", "seq", "pos", "selected")),
                               (selected, SELECTED, ("tables", "seq", "pos", "selected"))):
        for name in names:
            assert call(d, **{name: None}) == EINVAL, name
            assert call(d, **{name: P + (2 if name in loose else 4 if name == "mask" else 8)}) == EINVAL, name
        assert call(attn(n_tokens=0), ws=None, size=0, **{n: None for n in names}) == OK
    assert tree(d, words=0) == tree(d, words=5) == tree(attn(n_seqs=(1 << 20) + 1)) == ESHAPE
    assert select(d, budget=2) == select(d, first=-1) == select(d, recent=0) == select(d, budget=(1 << 20) + 1) == select(d, budget=2**31 - 1, recent=2**31 - 1) == EINVAL
    for big in (dict(n_tokens=(1 << 22) // 2), dict(max_blocks=(1 << 28) + 1), dict(n_kv_heads=(1 << 16) + 1, n_q_heads=(1 << 16) + 1)):
        assert select(attn(**big)) == selected(attn(**big)) == size_of("alora_block_select", attn(**big))[0] == ESHAPE, big
    for big in (dict(max_blocks=(1 << 26) + 1), dict(n_tokens=1 << 29), dict(n_tokens=1 << 24, n_q_heads=64, n_kv_heads=64, dtype=0), dict(n_tokens=1 << 24, n_q_heads=8, dtype=0)):
        assert tree(attn(**big)) == size_of("alora_tree_attention", attn(**big), 1)[0] == ESHAPE, big
    assert size_of("alora_block_select", attn(n_tokens=(1 << 21) - 1, max_blocks=1 << 28))[0] == size_of("alora_tree_attention", attn(max_blocks=1 << 26, n_tokens=1 << 22), 4)[0] == OK
    assert selected(d, budget=0) == selected(d, budget=(1 << 20) + 1) == EINVAL and selected(attn(block_size=1 << 20), budget=1 << 20) == ESHAPE
    assert size_of("alora_selected_attention", d, 0)[0] == EINVAL


def test_readers_refuse_workspaces():
    d = attn(n_slots=1 << 20, max_blocks=1 << 12)
    for call, entry, more in ((tree, "alora_tree_attention", (1,)), (select, "alora_block_select", ()), (selected, "alora_selected_attention", (64,))):
        s, n = size_of(entry, d, *more)
        kw = dict(budget=64) if call is selected else {}
        assert s == OK and n > 0
        assert call(d, ws=None, size=n, **kw) == call(d, ws=P + 8, size=n, **kw) == call(d, size=n - 1, **kw) == EWORKSPACE


def test_bounds_are_refused():
    def bounds(**kw):
        dims = {**dict(dtype=1, n_rows=5, n_kv_heads=2, head_dim=64, block_size=16, n_slots=160), **{k: v for k, v in kw.items() if k in dict(ab.AloraBoundsDims._fields_)}}
        a = [kw.get(n, P) for n in ("k", "slot", "bounds", "scales")]
        return ab.lib().alora_block_bounds(*a, ctypes.byref(ab.AloraBoundsDims(**dims)), None)
    for kw, status in ((dict(dtype=2), EINVAL), (dict(n_rows=-1), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(block_size=0), EINVAL), (dict(n_slots=-1), EINVAL),
                       (dict(head_dim=80), ESHAPE), (dict(n_slots=1 << 31), ESHAPE), (dict(n_kv_heads=1 << 17), ESHAPE), (dict(n_rows=(1 << 27) + 1), ESHAPE), (dict(k=None), EINVAL), (dict(slot=None), EINVAL),
                       (dict(bounds=None), EINVAL), (dict(scales=None), EINVAL), (dict(k=P + 8), EINVAL), (dict(slot=P + 4), EINVAL), (dict(bounds=P + 8), EINVAL),
                       (dict(scales=P + 2), EINVAL), (dict(n_rows=0, k=None), OK)):
        assert bounds(**kw) == status, kw
    assert ab.lib().alora_block_bounds(P, P, P, P, None, None) == EINVAL


def test_binding_refuses_what_it_would_misread():
    """Types, sizes, strides, and tensors on the host."""
    if torch.cuda.is_available():
        pytest.skip("tensors on the host stand in for the device's")
    i = lambda *n: torch.zeros(n, dtype=torch.int32)
    l = lambda *n: torch.zeros(n, dtype=torch.int64)
    args = [i(3), i(3), i(3), i(3), i(3, 4), i(7), i(6), i(3), i(6), i(4), i(9), i(9), i(9), l(9)]
    dims = ab.make_step_dims(args[4], 16, 9, args[5], 160)
    with pytest.raises(TypeError, match="on the GPU"):
        ab.alora_step_rows(*args, dims)
    for at, name in enumerate(("lengths", "change", "kept_blocks", "seq_adapters", "block_tables", "pool", "state", "lengths_out", "state_out", "row_offsets",
                               "token_seq_ids", "token_positions", "token_adapter_ids", "slot_mapping")):
        for bad in (args[at].float(), torch.cat([args[at]] * 2)):
            with pytest.raises((TypeError, ValueError), match=name):
                ab.alora_step_rows(*args[:at], bad, *args[at + 1:], dims)
    q, kv, bt = torch.zeros(5, 512), torch.zeros(64, 128), i(2, 4)
    attn = ab.make_attn_dims(q, kv, bt, 8, 2, 64, 16)
    good = dict(q=q, k_cache=kv, v_cache=kv, block_tables=bt, row_offsets=i(3), context_lens=i(2), tree_mask=l(5, 1), out=q.clone())
    for name, bad in (("q", q.bfloat16()), ("k_cache", kv.T), ("v_cache", kv[:32]), ("block_tables", bt.long()), ("row_offsets", i(2)), ("context_lens", i(3)),
                      ("tree_mask", i(5, 1)), ("tree_mask", l(4, 1)), ("out", q[:4])):
        with pytest.raises((TypeError, ValueError), match=name):
            ab.alora_tree_attention(**{**good, name: bad}, dims=attn, workspace=None)
    with pytest.raises((TypeError, ValueError), match="tree_parents"):
        ab.alora_tree_rows(i(4), i(3), i(2), l(5, 1), i(5))
    bounds, scales = torch.zeros(4, 2, 2, 64, dtype=torch.int8), torch.zeros(4, 2)
    sel = dict(q=q, bounds=bounds, scales=scales, block_tables=bt, token_seq_ids=i(5), token_positions=i(5), selected=i(5, 2, 3))
    for name, bad in (("bounds", bounds.float()), ("bounds", bounds[:3]), ("scales", scales.double()), ("token_seq_ids", i(4)), ("token_positions", l(5)), ("selected", i(5, 3))):
        with pytest.raises((TypeError, ValueError), match=name):
            ab.alora_block_select(**{**sel, name: bad}, n_first=1, n_recent=1, dims=attn, workspace=None)
    use = dict(q=q, k_cache=kv, v_cache=kv, block_tables=bt, token_seq_ids=i(5), token_positions=i(5), selected=i(5, 2, 3), out=q.clone())
    for name, bad in (("selected", l(5, 2, 3)), ("out", q.T), ("token_positions", i(3))):
        with pytest.raises((TypeError, ValueError), match=name):
            ab.alora_selected_attention(**{**use, name: bad}, dims=attn)
    bd = ab.make_bounds_dims(kv, l(6), 2, 64, 16)
    for name, bad in (("slot_mapping", i(6)), ("slot_mapping", l(5)), ("bounds", bounds[1:]), ("k_cache", kv.bfloat16())):
        with pytest.raises((TypeError, ValueError), match=name):
            ab.alora_block_bounds(**{**dict(k_cache=kv, slot_mapping=l(6), bounds=bounds, scales=scales), name: bad}, dims=bd)
