"""Refusals of the head and cache operators, found on the host before anything is launched (CPU; dummy addresses that nothing
dereferences), and the launches of calls, recorded without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2512_17910_amd import binding as ab

P = 0x100000
OK, EINVAL, ESHAPE, EWORKSPACE, EDATA = ab.ALORA_OK, ab.ALORA_EINVAL, ab.ALORA_ESHAPE, ab.ALORA_EWORKSPACE, ab.ALORA_EDATA


def heads_dims(**kw):
    d = dict(dtype=1, n_tokens=7, n_q_heads=4, n_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, norm=1, rope_positions=100, eps=1e-6,
             n_slots=64, q_stride=256, q_out_stride=256, k_stride=128, k_out_stride=128, v_stride=128, v_out_stride=128, dq_stride=0, dk_stride=0)
    d.update(kw)
    return ab.AloraHeadsDims(**d)


FORWARD = ("q", "q_out", "k", "kc", "v", "vc", "wq", "wk", "cos", "sin", "pos", "slot")


def forward(dims, **kw):
    a = {n: P for n in FORWARD}
    a["q_out"] = P + 0x1000
    a.update(kw)
    return ab.lib().alora_qk_norm_rope(*[a[n] for n in FORWARD], ctypes.byref(dims), None)


BACKWARD = ("q", "gq", "dq", "k", "gk", "dk", "wq", "wk", "dwq", "dwk", "cos", "sin", "pos")


def backward(dims, ws=P, size=1 << 24, **kw):
    a = {n: P + 0x1000 * i for i, n in enumerate(BACKWARD)}
    a.update(kw)
    return ab.lib().alora_qk_norm_rope_backward(*[a[n] for n in BACKWARD], ctypes.byref(dims), ws, size, None)


SHAPES = [(dict(dtype=3), EINVAL), (dict(n_tokens=-1), EINVAL), (dict(n_q_heads=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL),
          (dict(rotary_dim=-4), EINVAL), (dict(interleaved=2), EINVAL), (dict(norm=-1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
          (dict(eps=float("inf")), EINVAL), (dict(rope_positions=0), EINVAL), (dict(n_slots=-1), EINVAL), (dict(head_dim=60), ESHAPE),
          (dict(dtype=0, head_dim=66), ESHAPE), (dict(head_dim=264), ESHAPE), (dict(rotary_dim=62), ESHAPE), (dict(rotary_dim=68), ESHAPE),
          (dict(n_tokens=1 << 29), ESHAPE), (dict(n_q_heads=1 << 26), ESHAPE)]


@pytest.mark.parametrize("kw,status", SHAPES)
def test_shapes_are_refused(kw, status):
    d = heads_dims(**kw)
    n = ctypes.c_size_t(0)
    assert forward(d) == backward(d) == status
    assert ab.lib().alora_qk_norm_rope_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == status
    assert ab.lib().alora_qk_norm_rope_validate(P, P, ctypes.byref(d)) == status


def test_forward_arguments_are_refused():
    d = heads_dims()
    for name in ("q", "q_out", "kc", "vc", "wq", "wk", "cos", "sin", "pos", "slot"):
        assert forward(d, **{name: None}) == EINVAL, name
    for name in FORWARD:
        assert forward(d, **{name: P + (4 if name == "slot" else 2 if name == "pos" else 8)}) == EINVAL, name
    assert forward(heads_dims(norm=0)) == EINVAL and forward(heads_dims(rotary_dim=0)) == EINVAL       # weights, tables that no step takes
    for name, bad in (("q_stride", 248), ("q_out_stride", 257), ("k_stride", 120), ("k_out_stride", 132), ("v_stride", -128), ("v_out_stride", 1 << 41)):
        assert forward(heads_dims(**{name: bad})) == EINVAL, name
    assert forward(heads_dims(q_stride=264), q_out=P) == EINVAL                                        # in place, strides differ
    assert ab.lib().alora_qk_norm_rope(*[P] * 12, None, None) == EINVAL
    assert forward(heads_dims(n_tokens=0), q=None, q_out=None, kc=None, slot=None) == OK


def test_backward_arguments_are_refused():
    d = heads_dims()
    for name in BACKWARD:
        assert backward(d, **{name: None}) == EINVAL, name
        assert backward(d, **{name: P + (2 if name == "pos" else 8)}) == EINVAL, name
    for name, bad in (("q_stride", 248), ("q_out_stride", 257), ("k_stride", 120), ("k_out_stride", 132), ("dq_stride", 128), ("dk_stride", 64)):
        assert backward(heads_dims(**{name: bad})) == EINVAL, name
    large = heads_dims(n_tokens=3000)
    need = ab.alora_qk_norm_rope_workspace_bytes(large)
    assert need > 0 and need % (2 * 64 * 4) == 0
    assert backward(large, ws=None) == backward(large, ws=P + 8) == backward(large, size=need - 1) == EWORKSPACE
    assert ab.alora_qk_norm_rope_workspace_bytes(heads_dims(norm=0)) == 0 == ab.alora_qk_norm_rope_workspace_bytes(heads_dims(n_tokens=0))
    assert backward(heads_dims(norm=0, n_tokens=0), ws=None, size=0, wq=None, wk=None, dwq=None, dwk=None) == OK
    assert backward(heads_dims(q_out_stride=264), dq=P + 0x1000) == EINVAL                             # dq in dq_out's place, strides differ


def spec(**kw):
    d = dict(rotary_dim=64, scaling=2, base=1e4, factor=4.0, original=2048.0, low=1.0, high=32.0, magnitude=1.0)
    d.update(kw)
    return ab.AloraRopeSpec(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(scaling=3), EINVAL), (dict(base=0.0), EINVAL), (dict(base=float("nan")), EINVAL), (dict(base=float("inf")), EINVAL), (dict(factor=0.0), EINVAL),
    (dict(factor=float("inf")), EINVAL), (dict(original=0.0), EINVAL), (dict(low=32.0), EINVAL), (dict(high=float("nan")), EINVAL),
    (dict(magnitude=float("inf")), EINVAL), (dict(rotary_dim=0), ESHAPE), (dict(rotary_dim=7), ESHAPE), (dict(rotary_dim=514), ESHAPE)])
def test_rope_specs_are_refused(kw, status):
    assert ab.lib().alora_rope_tables(P, P, 0, 8, ctypes.byref(spec(**kw)), None) == status


def test_rope_table_arguments_are_refused():
    f = lambda cos=P, sin=P, first=0, rows=8, s=spec(): ab.lib().alora_rope_tables(cos, sin, first, rows, None if s is None else ctypes.byref(s), None)
    assert f(cos=None) == f(sin=None) == f(cos=P + 4) == f(first=-1) == f(rows=-1) == f(s=None) == EINVAL
    assert f(first=1 << 24, rows=1) == f(rows=(1 << 24) + 1) == f(first=1 << 62) == ESHAPE
    assert f(rows=0, cos=None, sin=None) == OK
    # what the scaling does not take is not looked at
    assert f(rows=0, s=spec(scaling=0, factor=0.0, original=0.0)) == OK
    with pytest.raises(ValueError):
        ab.make_rope_spec(64, scaling="other")
    with pytest.raises(ValueError):
        ab.alora_rope_tables(torch.zeros(4, 31), torch.zeros(4, 31), ab.make_rope_spec(64))


def cache_dims(n_layers=2, ptr=P, **kw):
    d = dict(dtype=1, n_layers=n_layers, n_kv_heads=2, head_dim=64, block_size=16, n_slots=256)
    d.update(kw)
    tab = (ctypes.c_void_p * max(1, n_layers))(*[ptr] * n_layers)
    c = ab.AloraCacheDims(**d, k_caches=ctypes.cast(tab, ctypes.c_void_p), v_caches=ctypes.cast(tab, ctypes.c_void_p))
    c.keep = tab
    return c


def copy(src, dst, dims=None, n=None):
    s, d = (None if x is None else np.array(x, np.int32) for x in (src, dst))
    dims = dims or cache_dims()
    return ab.lib().alora_cache_copy_blocks(None if s is None else s.ctypes.data, None if d is None else d.ctypes.data, len(s) if n is None else n,
                                            ctypes.byref(dims), None)


def move(dims=None, n=3, rot=64, pos=10, il=0, **kw):
    a = dict(src=P, dst=P, shift=P, cos=P, sin=P)
    a.update(kw)
    dims = dims or cache_dims()
    return ab.lib().alora_cache_move_rows(a["src"], a["dst"], a["shift"], n, a["cos"], a["sin"], pos, rot, il, ctypes.byref(dims), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), EINVAL), (dict(n_layers=-1), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(block_size=0), EINVAL),
    (dict(n_slots=-16), EINVAL), (dict(head_dim=60), ESHAPE), (dict(head_dim=264), ESHAPE), (dict(n_slots=250), ESHAPE), (dict(n_layers=4097), ESHAPE),
    (dict(n_slots=1 << 50), ESHAPE), (dict(block_size=1 << 24, n_slots=1 << 24), ESHAPE), (dict(ptr=None), EINVAL), (dict(ptr=P + 8), EINVAL)])
def test_caches_are_refused(kw, status):
    if kw.get("n_layers") == -1:
        d = cache_dims(1)
        d.n_layers = -1
    else:
        d = cache_dims(**kw)
    assert copy([0], [1], d) == move(d) == status
    if "ptr" not in kw:
        assert ab.lib().alora_cache_move_rows_validate(P, P, P, 3, 10, ctypes.byref(d)) == status


@pytest.mark.parametrize("n,blocks", [(0, 200), (30, 200), (30, 1 << 20)])      # (short and long lists, of small and large pools, are checked in different ways)
def test_lists_of_blocks_are_refused(n, blocks):
    fill = lambda a, first: a + list(range(first, first + n))
    d = cache_dims(n_slots=16 * blocks)
    for src, dst in (([0, blocks], [1, 2]), ([0, -2], [1, 2]), ([0, 1], [3, blocks]), ([0, 1], [3, -1]), ([0, 1], [3, 3]), ([0, 1], [1, 2]), ([5, 1], [5, 2]),
                     ([-1, -1], [4, 4]), ([-1, 4], [4, 6])):
        assert copy(fill(src, 40), fill(dst, 100), d) == EDATA, (src, dst)
    assert copy(None, [1], d, 1) == copy([1], None, d, 1) == copy([1], [2], d, -1) == EINVAL
    assert copy([], [], d) == OK and copy([1], [2], cache_dims(0)) == OK
    assert copy([0], [1], cache_dims(n_slots=0)) == EDATA


def test_move_arguments_are_refused():
    for name in ("src", "dst", "shift", "cos", "sin"):
        assert move(**{name: None}) == EINVAL, name
        assert move(**{name: P + (2 if name == "shift" else 4)}) == EINVAL, name
    assert move(n=-1) == move(rot=-4) == move(il=2) == move(pos=0) == move(rot=0) == EINVAL
    assert move(rot=62) == move(rot=68) == move(n=(1 << 24) + 1) == ESHAPE
    assert move(n=0) == move(dims=cache_dims(0)) == move(n=0, src=None, dst=None, shift=None) == OK


def test_binding_refuses_what_it_would_misread():
    t = lambda *s: torch.zeros(*s)
    q, k = t(4, 128), t(32, 64)
    rope = (t(10, 16), t(10, 16))
    ok = ab.make_heads_dims(q, q, None, k, 4, 2, 32, rope=rope)
    assert (ok.rotary_dim, ok.q_stride, ok.k_stride, ok.k_out_stride, ok.rope_positions, ok.n_slots) == (32, 128, 0, 64, 10, 32)
    for bad in (lambda: ab.make_heads_dims(q, q, None, k, 4, 2, 64, rope=rope), lambda: ab.make_heads_dims(q.t(), q, None, k, 4, 2, 32),
                lambda: ab.make_heads_dims(q, q.bfloat16(), None, k, 4, 2, 32), lambda: ab.make_heads_dims(q, q[:2], None, k, 4, 2, 32),
                lambda: ab.make_heads_dims(q, q, None, k, 4, 2, 32, rope=(rope[0].double(), rope[1])),
                lambda: ab.make_heads_dims(q, q, None, k, 4, 2, 32, rope=(rope[0], rope[1][:9])),
                lambda: ab.make_heads_dims(q, q, k[:4], k, 4, 2, 32, v=k[:4], v_out=k[:20]),
                lambda: ab.make_cache_dims([k], [k[:16]], 2, 32, 16), lambda: ab.make_cache_dims([], [], 2, 32, 16),
                lambda: ab.make_cache_dims([k], [k, k], 2, 32, 16), lambda: ab.make_cache_dims([k.t()], [k.t()], 2, 32, 16),
                lambda: ab.alora_cache_copy_blocks(np.zeros(2, np.int64), np.ones(2, np.int32), ab.make_cache_dims([k], [k], 2, 32, 16)),
                lambda: ab.alora_cache_copy_blocks(np.zeros(2, np.int32), np.ones(1, np.int32), ab.make_cache_dims([k], [k], 2, 32, 16)),
                lambda: ab.alora_cache_move_rows(torch.zeros(2).long(), torch.zeros(3).long(), None, None, ab.make_cache_dims([k], [k], 2, 32, 16)),
                lambda: ab.alora_qk_norm_rope_backward(q, q, t(4, 256)[:, :128], k[:4], k[:4], k[:4], None, None, None, None, rope, None,
                                                       ab.make_heads_dims(q, q, k[:4], k[:4], 4, 2, 32, rope=rope, norm=False))):
        with pytest.raises(ValueError):
            bad()
    dims = ab.make_cache_dims([k], [k], 2, 32, 16)
    some = np.arange(4, dtype=np.int32)
    with pytest.raises(ValueError):
        ab.alora_cache_copy_blocks(some[::2], some[:2], dims)
    ab._host_int32(some[:0], "src"), ab._host_int32(np.zeros(0, np.int32), "src")      # (an empty array's strides say nothing)
    some.flags.writeable = False
    assert ab._host_int32(some, "src") == some.ctypes.data and ab._host_int32(some[1:].copy(), "src") != some.ctypes.data
    for bad in (lambda: ab.alora_qk_norm_rope(q, q, None, k, None, None, None, None, rope, torch.zeros(4).long(), torch.zeros(4).long(), ok),
                lambda: ab.alora_qk_norm_rope(q, q, None, k, None, None, None, None, rope, torch.zeros(4).int(), torch.zeros(4).int(), ok),
                lambda: ab.alora_qk_norm_rope_backward(q, q, q, k[:4], k[:4], k[:4], None, None, None, None, rope, torch.zeros(4).long(),
                                                       ab.make_heads_dims(q, q, k[:4], k[:4], 4, 2, 32, rope=rope, norm=False)),
                lambda: ab.alora_cache_move_rows(torch.zeros(2).int(), torch.zeros(2).int(), None, None, dims),
                lambda: ab.alora_cache_move_rows(torch.zeros(4).long()[::2], torch.zeros(2).long(), None, None, dims),
                lambda: ab.alora_cache_move_rows(torch.zeros(2).long(), torch.zeros(2).long(), torch.zeros(2).long(), rope, dims)):
        with pytest.raises(TypeError):
            bad()
    one = ab.make_heads_dims(q[:1], q[:1], None, k, 4, 2, 32)
    assert one.q_stride >= 128


# ---- tensors of a call that its description does not know: refused in the binding, where they would be misread ---------------------------
def heads_call(dtype=None, back=False, **kw):
    """A call of 4 rows, 4 / 2 heads of 32, all right but for what kw says (on the CPU: what is right is refused last, as no device tensor)."""
    dtype = dtype or torch.bfloat16
    q, k = torch.zeros(4, 128, dtype=dtype), torch.zeros(32, 64, dtype=dtype)
    rope = (torch.zeros(10, 16), torch.zeros(10, 16))
    a = dict(wq=torch.ones(32, dtype=dtype), wk=torch.ones(32, dtype=dtype), rope=rope, pos=torch.zeros(4, dtype=torch.int32), slot=torch.arange(4),
             dwq=torch.zeros(32), dwk=torch.zeros(32))
    a.update(kw)
    if back:
        dims = ab.make_heads_dims(q, q, k[:4], k[:4], 4, 2, 32, rope=rope)
        ab.alora_qk_norm_rope_backward(q, q, q, k[:4], k[:4], k[:4], a["wq"], a["wk"], a["dwq"], a["dwk"], a["rope"], a["pos"], dims)
    else:
        ab.alora_qk_norm_rope(q, q, None, k, None, None, a["wq"], a["wk"], a["rope"], a["pos"], a["slot"], ab.make_heads_dims(q, q, None, k, 4, 2, 32, rope=rope))


@pytest.mark.parametrize("back", [False, True])
def test_norm_weights_of_another_type_or_size_are_refused(back):
    bf, f = torch.bfloat16, torch.float32
    for dtype, w in ((bf, torch.ones(32)), (f, torch.ones(32, dtype=bf)), (bf, torch.ones(32, dtype=torch.float16)), (f, torch.ones(32).double()),
                     (bf, torch.ones(16))):
        for name in ("wq", "wk"):
            with pytest.raises(TypeError, match=name):
                heads_call(dtype, back, **{name: w})
    for dtype, w in ((bf, torch.ones(16, dtype=bf)), (f, torch.ones(31)), (f, torch.ones(64)[::2]), (f, torch.ones(1).expand(32)), (f, torch.ones(128))):
        for name in ("wq", "wk"):
            with pytest.raises(ValueError, match=name):
                heads_call(dtype, back, **{name: w})


def test_gradients_of_norm_weights_of_another_type_or_size_are_refused():
    for name in ("dwq", "dwk"):
        for w in (torch.zeros(32, dtype=torch.int32), torch.zeros(32, dtype=torch.bfloat16), torch.zeros(32).double()):
            with pytest.raises(TypeError, match=name):
                heads_call(back=True, **{name: w})
        for w in (torch.zeros(31), torch.zeros(64)[::2], torch.zeros(8)):
            with pytest.raises(ValueError, match=name):
                heads_call(back=True, **{name: w})


@pytest.mark.parametrize("back", [False, True])
def test_positions_and_slots_that_are_not_dense_integers_of_every_row_are_refused(back):
    i32, i64 = torch.int32, torch.int64
    for name, kinds in (("token_positions", (torch.float32, torch.uint8, i64)), ("slot_mapping", (torch.float64, i32))):
        key = dict(token_positions="pos", slot_mapping="slot")[name]
        if back and key == "slot":
            continue
        for kind in kinds:
            with pytest.raises(TypeError, match=name):
                heads_call(back=back, **{key: torch.zeros(4, dtype=kind)})
        right = i32 if key == "pos" else i64
        for t in (torch.zeros(8, dtype=right)[::2], torch.zeros(3, dtype=right), torch.zeros(1, dtype=right).expand(4)):
            with pytest.raises(ValueError, match=name):
                heads_call(back=back, **{key: t})


@pytest.mark.parametrize("back", [False, True])
def test_tables_that_are_not_those_of_the_call_are_refused(back):
    z = torch.zeros
    for rope in ((z(10, 16).bfloat16(), z(10, 16)), (z(10, 16), z(10, 16).double()), (z(10, 32)[:, ::2], z(10, 16)), (z(10, 16), z(9, 16)), (z(9, 16), z(9, 16)),
                 (z(10, 8), z(10, 8)), (z(160), z(160)), (z(16, 10).t(), z(16, 10).t())):
        with pytest.raises(ValueError, match="rope"):
            heads_call(back=back, rope=rope)


def test_tables_of_moved_rows_are_checked():
    z, k = torch.zeros, torch.zeros(32, 64)
    dims = ab.make_cache_dims([k], [k], 2, 32, 16)
    src, dst, shift = torch.arange(3), torch.arange(8, 11), torch.ones(3, dtype=torch.int32)
    for rope in ((z(10, 16).half(), z(10, 16)), (z(10, 16).bfloat16(), z(10, 16).bfloat16()), (z(10, 16), z(3, 32)[:, ::2]), (z(10, 16), z(10, 8)), (z(10, 16), z(9, 16)),
                 (z(160), z(160))):
        with pytest.raises(ValueError, match="rope"):
            ab.alora_cache_move_rows(src, dst, shift, rope, dims)


def test_lists_of_rows_that_are_not_dense_integers_are_refused():
    z, k = torch.zeros, torch.zeros(32, 64)
    dims, rope = ab.make_cache_dims([k], [k], 2, 32, 16), (z(10, 16), z(10, 16))
    src, dst, shift = torch.arange(3), torch.arange(8, 11), torch.ones(3, dtype=torch.int32)
    for call in (lambda s, d, h: ab.alora_cache_move_rows(s, d, h, rope, dims), lambda s, d, h: ab.alora_cache_move_rows_validate(s, d, h, rope, dims)):
        for name, lists in (("src", (src.double(), dst, shift)), ("dst", (src, dst.double(), shift)), ("shift", (src, dst, shift.float()))):
            with pytest.raises(TypeError, match=name):
                call(*lists)
        with pytest.raises(TypeError, match="shift"):
            call(src, dst, torch.ones(6, dtype=torch.int32)[::2])
        for lists in ((src, dst[:2], shift), (src, dst, shift[:2])):
            with pytest.raises(ValueError):
                call(*lists)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_host_tensors_are_refused(dtype):
    """Their addresses would go to a kernel.  (All else about these calls is right.)"""
    dtype = getattr(torch, dtype)
    for back in (False, True):
        with pytest.raises(TypeError, match="on the GPU"):
            heads_call(dtype, back)
    k = torch.zeros(32, 64, dtype=dtype)
    dims, src, dst = ab.make_cache_dims([k], [k], 2, 32, 16), torch.arange(3), torch.arange(8, 11)
    for shift, rope in ((None, None), (torch.ones(3, dtype=torch.int32), (torch.zeros(10, 16), torch.zeros(10, 16)))):
        with pytest.raises(TypeError, match="on the GPU"):
            ab.alora_cache_move_rows(src, dst, shift, rope, dims)
    with pytest.raises(TypeError, match="on the GPU"):
        ab.alora_cache_copy_blocks(np.zeros(1, np.int32), np.ones(1, np.int32), dims)
    with pytest.raises(TypeError, match="on the GPU"):
        ab.alora_rope_tables(torch.zeros(4, 16), torch.zeros(4, 16), ab.make_rope_spec(32))


# ---- launches, recorded without a GPU (see launch_recorder.c) -------------------------------------
RECORD = """
import ctypes, json, re, sys, types
sys.modules["torch"] = types.ModuleType("torch")         # (the real one would register kernels of its own)
rec = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)      # ahead of the library: its HIP calls bind here
sys.path[:0] = sys.argv[2:4]
import test_operators_abi as t
from launches import _Launch
t.ab._lib = t.ab.lib()
rec.rec_get.restype = ctypes.POINTER(_Launch)
out = []
for name, args in json.load(sys.stdin):
    rec.rec_reset()
    status = getattr(t, name)(*args)
    launches = []
    for i in range(rec.rec_count()):
        r = rec.rec_get(i).contents
        m = re.search(r"N5alora(\\d+)", r.name.decode())
        launches.append([r.name.decode()[m.end():m.end() + int(m.group(1))], list(r.grid), list(r.block)])
    out.append([status, launches])
print(json.dumps(out))
"""


def record_forward(kw, has_v):
    d = heads_dims(**kw)
    return forward(d, **({} if has_v else dict(v=None, vc=None, k=None)))


def record_backward(kw):
    return backward(heads_dims(**kw))


def record_copy(n, layers, blocks):
    return copy(list(range(n)), list(range(n, 2 * n)), cache_dims(layers, n_slots=16 * blocks))


def record_move(n, layers, rot, heads):
    d = cache_dims(layers, n_kv_heads=heads)
    return move(d, n=n, rot=rot, **({} if rot else dict(shift=None, cos=None, sin=None)))


def test_launches_of_calls(tmp_path):
    import json
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    rec = str(tmp_path / "librec.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", "-o", rec, os.path.join(here, "launch_recorder.c")], check=True)

    def run(*calls):
        r = subprocess.run([sys.executable, "-c", RECORD, rec, here, os.path.dirname(here)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-3000:]
        out = json.loads(r.stdout)
        assert all(s == OK for s, _ in out), out
        return [launches for _, launches in out]

    wide = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, rotary_dim=128, q_stride=4096, q_out_stride=4096, k_stride=1024, k_out_stride=1024,
                v_stride=1024, v_out_stride=1024)
    one, small, many, full = run(["record_forward", [dict(wide, n_tokens=1), False]], ["record_forward", [dict(n_tokens=100), True]],
                                 ["record_forward", [dict(wide, n_tokens=(1 << 20) + 5), True]], ["record_forward", [dict(wide, n_tokens=2000), True]])
    assert one == [["heads_kernel", [1, 1, 1], [5 * 64, 1, 1]]]                 # four units of queries, one of keys
    # rows of 4 / 2 heads of 64 (16 heads a wavefront): 4 and 8 rows on one, 8 rows of values
    assert small == [["heads_packed_kernel", [-(-(25 + 13 + 13) // 4), 1, 1], [256, 1, 1]]]
    # three wavefronts of two units (the last of one) and one of values
    assert many == [["heads_kernel", [1 << 20, 2, 1], [4 * 64, 1, 1]]] and full == [["heads_kernel", [2000, 1, 1], [4 * 64, 1, 1]]]
    few, back, plain = run(["record_backward", [dict(wide, n_tokens=9)]], ["record_backward", [dict(wide, n_tokens=4096)]], ["record_backward", [dict(n_tokens=0)]])
    assert [l[0] for l in few] == ["heads_back_kernel"] and few[0][1] == [1, 1, 1]
    assert [l[:2] for l in back] == [["heads_back_kernel", [256, 1, 1]], ["heads_weights_kernel", [16, 1, 1]]] and back[0][2] == [15 * 64, 1, 1]
    assert [l[0] for l in plain] == ["heads_weights_kernel"]
    short, pairs, layers = run(["record_copy", [3, 2, 20]], ["record_copy", [353, 2, 1000]], ["record_copy", [1, 65, 20]])
    assert short == [["copy_blocks_kernel", [1, 3, 4], [256, 1, 1]]]            # 16 rows of 2 heads of 64: 4 KiB
    assert [l[1] for l in pairs] == [[1, 352, 4], [1, 1, 4]] and [l[1] for l in layers] == [[1, 1, 128], [1, 1, 2]]
    turned, copied, wide_rows = run(["record_move", [100, 65, 64, 2]], ["record_move", [100, 1, 0, 2]], ["record_move", [100, 1, 64, 80]])
    # two heads of 64: 8 rows of a wavefront either way; 80 heads: 5 wavefronts of turned keys a row
    assert [l[1] for l in turned] == [[4, 128, 1], [4, 2, 1]] and copied == [["move_rows_kernel", [4, 2, 1], [256, 1, 1]]]
    assert wide_rows[0][1] == [125, 2, 1]


def record_calls(tmp_path, *calls):
    """(status, launches) of calls of the record_ functions above, in a process without a GPU."""
    import json
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    rec = str(tmp_path / "librec.so")
    subprocess.run(["gcc", "-O1", "-w", "-shared", "-fPIC", "-o", rec, os.path.join(here, "launch_recorder.c")], check=True)
    r = subprocess.run([sys.executable, "-c", RECORD, rec, here, os.path.dirname(here)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout)


def test_rows_of_few_heads_fill_a_grid_of_fewer_than_2_to_32_threads(tmp_path):
    """Heads of 256 on 16 lanes: four rows of one query head, two of two K/V heads and two of their values to a wavefront, 1.25 of them a row.  A dimension of a
    grid holds fewer than 2^32 threads: 2^26 wavefronts are one too many, whatever the last workgroup leaves empty."""
    few = dict(n_q_heads=1, n_kv_heads=2, head_dim=256, rotary_dim=256, q_stride=256, q_out_stride=256, k_stride=512, k_out_stride=512, v_stride=512, v_out_stride=512)
    items = lambda T: -(-T // 4) + 2 * -(-T // 2)
    most = max(T for T in range(53687080, 53687100) if items(T) <= (1 << 26) - 4)
    rows = [1000, most - 1, most, most + 1, most + 2, most + 3, most + 4, most + 5, most + 30]
    assert any((1 << 26) - 4 < items(T) < 1 << 26 for T in rows)
    for T, (status, launches) in zip(rows, record_calls(tmp_path, *[["record_forward", [dict(few, n_tokens=T), True]] for T in rows])):
        assert status == OK and len(launches) == 1
        (name, grid, block), = launches
        assert all(g * b < 1 << 32 for g, b in zip(grid, block)), (T, launches)
        assert name == ("heads_packed_kernel" if T <= most else "heads_kernel"), (T, launches)
        if T <= most:
            assert grid[0] == -(-items(T) // 4)


def test_rows_of_two_gibibytes_and_more(tmp_path):
    """Values are copied in pieces of 2 KiB; their bytes leave 31 bits behind in fp32 rows of 2^29 features and more, the widest there are."""
    wide = lambda hkv, d: dict(dtype=0, n_tokens=1, n_q_heads=1, n_kv_heads=hkv, head_dim=d, rotary_dim=4, q_stride=d, q_out_stride=d, k_stride=hkv * d,
                               k_out_stride=hkv * d, v_stride=hkv * d, v_out_stride=hkv * d)
    sizes = [(1 << 21, 256), ((1 << 21) - 1, 256), ((1 << 22) - 1, 256), ((1 << 28) - 1, 4), ((1 << 27) + 5, 4)]
    for size, (status, launches) in zip(sizes, record_calls(tmp_path, *[["record_forward", [wide(*size), True]] for size in sizes])):
        assert status == OK and launches == [["heads_kernel", [1, 1, 1], [8 * 64, 1, 1]]], (size, launches)


def test_pieces_of_values_cover_the_widest_rows_in_32_bits():
    """What heads_kernel computes of a lane's piece of the values' row, in unsigned 32 bits, for rows of up to 2^32 - 16 bytes."""
    u = lambda x: x & 0xffffffff
    for v_bytes in (16, 2048, 2064, (1 << 31) - 16, 1 << 31, (1 << 32) - 4096, (1 << 32) - 2048, (1 << 32) - 1040, (1 << 32) - 16):
        pieces = u(v_bytes - 1) // 2048 + 1
        for piece in {0, 1, pieces // 2, pieces - 2, pieces - 1} & set(range(pieces)):
            covered = set()
            for lane in range(64):
                o = u(piece * 2048 + lane * 16)
                covered |= {x for x in (o, u(o + 1024)) if x < v_bytes}
            assert covered == set(range(2048 * piece, min(v_bytes, 2048 * piece + 2048), 16)), (v_bytes, piece)


# ---- every instantiation of the kernels of heads: sizes that test_gpu_operators.py runs -----------------------------------------------
# (type, head_dim, rotary_dim, neighbours): one for each layout of a head on lanes
LAYOUTS = [("bf16", 32, 32, False), ("bf16", 80, 8, False), ("bf16", 64, 4, False), ("bf16", 96, 24, True), ("bf16", 64, 20, True),
           ("f32", 80, 20, False), ("f32", 48, 4, False), ("f32", 64, 64, True)]


def heads_of_a_layout(dtype, d, rot, il, units_q, units_k):
    """(query heads, K/V heads) that fill so many units of 64 lanes, the last of each in part."""
    bf16 = dtype == "bf16"
    if il:
        V = 8 if bf16 and rot % 8 == 0 else 4
        lanes = (d // V + 1) // 2
    else:
        V = 8 if bf16 else 4
        while V > 2 and (0 < rot // 2 < V or 0 < d - rot < V):
            V //= 2
        lanes = -(-rot // 2 // V) + (-(-(d - rot) // V) + 1) // 2
    per = 64 >> (lanes - 1).bit_length()
    return units_q * per - (per > 1), units_k * per - (per > 2)


# (rows, units of queries, units of keys): one, two (one left over) and three units of a wavefront
UNITS = {1: (70, 4, 2), 2: (1700, 3, 2), 3: (1400, 4, 2)}


def record_layout(back, dtype, d, rot, il, norm, T, hq, hkv):
    w, e = hq * d, hkv * d
    dims = heads_dims(dtype=1 if dtype == "bf16" else 0, n_tokens=T, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, rotary_dim=rot, interleaved=int(il), norm=int(norm),
                      q_stride=w, q_out_stride=w, k_stride=e, k_out_stride=e, v_stride=e, v_out_stride=e, n_slots=T)
    none = {} if norm else dict(wq=None, wk=None)
    return backward(dims, **none, **({} if norm else dict(dwq=None, dwk=None))) if back else forward(dims, **none)


RECORD_INTS = RECORD.replace("list(r.block)]", "[int(v) for v in re.findall(r'L[ib](\\d+)E', r.name.decode())]]")


def test_the_cases_run_on_the_gpu_reach_every_instantiation(tmp_path, monkeypatch):
    monkeypatch.setitem(globals(), "RECORD", RECORD_INTS)
    calls, want = [], []
    for dtype, d, rot, il in LAYOUTS:
        for norm in (True, False):
            for units, (T, uq, uk) in UNITS.items():
                calls.append(["record_layout", [False, dtype, d, rot, il, norm, T, *heads_of_a_layout(dtype, d, rot, il, uq, uk)]])
            calls.append(["record_layout", [False, dtype, d, rot, il, norm, 333, 2, 1]])
            calls.append(["record_layout", [True, dtype, d, rot, il, norm, 333, *heads_of_a_layout(dtype, d, rot, il, 4, 2)]])
    got = {"heads_kernel": set(), "heads_packed_kernel": set(), "heads_back_kernel": set()}
    for call, (status, launches) in zip(calls, record_calls(tmp_path, *calls)):
        assert status == OK
        name, grid, ints = launches[0]
        assert ints[0] == (call[1][1] == "bf16") and ints[2] == call[1][4] and ints[3] == call[1][5], (call, launches)
        got[name].add(tuple(ints))
    layouts = {(1, 8, 0), (1, 4, 0), (1, 2, 0), (1, 8, 1), (1, 4, 1), (0, 4, 0), (0, 2, 0), (0, 4, 1)}
    normed = {(*l, n) for l in layouts for n in (0, 1)}
    assert got["heads_kernel"] == {(*l, u) for l in normed for u in (1, 2, 3)}
    assert got["heads_packed_kernel"] == got["heads_back_kernel"] == normed


def test_lists_of_blocks_are_checked_on_both_sides_of_the_rule():
    """30 blocks: up to 128 words of bits for each the pool's bits, from there on the sorted list."""
    for blocks in (30 * 64 * 128, 30 * 64 * 129):
        d = cache_dims(n_slots=16 * blocks)
        src, dst = list(range(30)), [blocks - 1 - i for i in range(30)]
        for i, value in ((3, dst[4]), (29, dst[0])):
            assert copy(src, dst[:i] + [value] + dst[i + 1:], d) == EDATA       # named twice
            assert copy(src[:i] + [value] + src[i + 1:], dst, d) == EDATA       # source and destination


def test_host_lists_in_another_byte_order_are_refused():
    k = torch.zeros(32, 64)
    dims, one = ab.make_cache_dims([k], [k], 2, 32, 16), np.ones(1, np.int32)
    for src, dst in ((one.astype(">i4"), one), (one, one.astype(">i4"))):
        with pytest.raises(ValueError, match="int32"):
            ab.alora_cache_copy_blocks(src, dst, dims)
